"""A decoder's serving operators on the GPU against plain implementations: the paged 8-bit cache (codes and scales bit for bit by the formula in
separately rounded fp32, and near the value in 64 bits), attention over it and drawing tokens (64 bits)."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

INT8, E4M3 = 0, 1
TOP = {INT8: np.float32(127), E4M3: np.float32(448)}


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a HIP device"
    return t


@pytest.fixture(scope="module")
def ops():
    from paper_2107_06469_amd import ops as o
    return o


def e4m3_values():
    """What the 256 codes stand for."""
    c = np.arange(256)
    s, e, m = np.where(c >> 7, -1.0, 1.0), (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v[(c & 127) == 127] = np.nan
    return s * v


E4M3_VALUES = e4m3_values()


def values(codes, kind):
    return codes.view(np.int8).astype(np.float64) if kind == INT8 else E4M3_VALUES[codes]


def to_codes(x, kind):
    """fp32 values already divided by the scale -> codes."""
    x = np.where(np.isnan(x), np.float32(0), np.clip(x, -TOP[kind], TOP[kind])).astype(np.float32)
    if kind == INT8:
        return np.rint(x).astype(np.int8).view(np.uint8)
    a = np.abs(x).astype(np.float64)
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.where(a > 0, a, 1))), -6) - 3)
    a = np.rint(a / step) * step                     # exact: a has 24 bits, the quotient is below 16
    table = E4M3_VALUES[:127]
    return (np.searchsorted(table, a) | (np.signbit(x) << 7)).astype(np.uint8)


def bf16(x):
    """fp32 -> the nearest bf16, as fp32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)


def turn(x, cs, rot, rot_dim):
    """x [heads, DH] fp32, cs [rot_dim]; every product and sum rounded by itself."""
    if not rot:
        return x
    x, h = x.copy(), rot_dim // 2
    c, s = cs[:h], cs[h:]
    a, b = (slice(0, h), slice(h, rot_dim)) if rot == 1 else (slice(0, rot_dim, 2), slice(1, rot_dim, 2))
    u, v = x[:, a].copy(), x[:, b].copy()
    x[:, a], x[:, b] = u * c - v * s, v * c + u * s
    return x


class Setup:
    """A cache of G models with random contents, a page table that jumps about the pool, and a call's tokens."""

    def __init__(self, torch, ops, kind, G, HKV, DH, page, new, total, seed, spare=0, one=False):
        r = np.random.default_rng(seed)
        self.torch, self.ops, self.kind, self.G, self.HKV, self.DH, self.page, self.r = torch, ops, kind, G, HKV, DH, page, r
        self.new, self.total, self.B = list(new), list(total), len(new)
        need = [-(-t // page) for t in total]
        self.n_pages, self.max_pages = sum(need) + 2, max(max(need), 1)
        ids = r.permutation(self.n_pages)
        self.table = r.integers(-5, self.n_pages + 5, size=(self.B, self.max_pages)).astype(np.int32)   # unused entries: anything
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = ids[at:at + n]
            at += n
        self.ptr = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.n_tok = int(self.ptr[-1])
        shape = (self.n_pages, HKV, page, DH)
        # anything in the slots, NaN codes among them; what is read of it is drawn below
        self.k, self.v = ([r.integers(0, 256, size=shape).astype(np.uint8) for _ in range(G)] for _ in range(2))
        self.ks, self.vs = ([(0.02 * np.exp(r.normal(size=shape[:2]))).astype(np.float32) for _ in range(G)] for _ in range(2))
        for pool in (*self.k, *self.v):
            for b in range(self.B):
                for t in range(total[b]):
                    x = r.normal(size=(HKV, DH)) * (TOP[kind] / 3)
                    pool[self.table[b, t // page], :, t % page] = to_codes(x.astype(np.float32), kind)
        self.spare = spare
        self.dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        big = [[torch.full((self.n_pages, HKV * page * DH + spare), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(G)] for _ in range(2)]
        self.pools = [[t[:, :HKV * page * DH].view(shape) if not spare else t.as_strided(shape, (HKV * page * DH + spare, page * DH, DH, 1)) for t in two]
                      for two in big]
        for pools, host in zip(self.pools, (self.k, self.v)):
            for t, h in zip(pools, host):
                t.copy_(self.dev(h))
        self.scales = [[self.dev(s) for s in two] for two in (self.ks, self.vs)]
        self.cache = ops.Cache(kind, *self.pools, *self.scales, self.dev(self.table))
        self.lens = self.dev(np.array(total, dtype=np.int32))
        self.call = dict(q_ptr=None if one else self.dev(self.ptr), n_tok=self.n_tok, max_q=max(max(self.new), 1), max_len=max(max(total), 1))

    def bf16(self, *shape, scale=1.0):
        x = bf16(self.r.normal(size=shape) * scale)
        return x, self.dev(x).to(self.torch.bfloat16)


def check_append(torch, ops, kind, G, H, HKV, DH, page, new, total, rot, rot_dim, seed, spare=0, one=False, in_place=False, poison=False, pad=0,
                 times=1):
    s = Setup(torch, ops, kind, G, HKV, DH, page, new, total, seed, spare, one)
    width = (H + 2 * HKV) * DH
    ld = width + pad
    angle = np.arange(s.call["max_len"])[:, None] * 100.0 ** (-np.arange(max(rot_dim // 2, 1))[None] / max(rot_dim // 2, 1))
    cs = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    host, dev = zip(*(s.bf16(s.n_tok, ld, scale=3.0) for _ in range(G)))
    if poison:
        for h, d in zip(host, dev):
            for n, what in enumerate((np.nan, np.inf, -np.inf, 0.0)):
                h[n % s.n_tok, n::97] = what
            d.copy_(s.dev(h))
    q = list(dev) if in_place else [torch.full((s.n_tok, H * DH + pad), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(G)]
    for _ in range(times):
        ops.hydra_op_cache_append(s.cache, s.lens, H, ld, ld if in_place else H * DH + pad, list(dev), q, rot=rot, rot_dim=rot_dim,
                                  cos_sin=s.dev(cs) if rot else None, **s.call)
    torch.cuda.synchronize()
    least = np.float32(2.0 ** -126)
    for g in range(G):
        want_q = np.zeros((s.n_tok, H * DH), dtype=np.float32)
        pools, scales = [s.k[g].copy(), s.v[g].copy()], [s.ks[g].copy(), s.vs[g].copy()]
        for b in range(s.B):
            n, pos0 = s.new[b], s.total[b] - s.new[b]
            rows = host[g][s.ptr[b]:s.ptr[b + 1], :width].reshape(n, H + 2 * HKV, DH)
            with np.errstate(invalid="ignore"):
                x = np.stack([np.concatenate([turn(rows[j, :H + HKV], cs[pos0 + j], rot, rot_dim), rows[j, H + HKV:]]) for j in range(n)]) if n else rows
            want_q[s.ptr[b]:s.ptr[b + 1]] = x[:, :H].reshape(n, H * DH)
            for pool, scale, y in zip(pools, scales, (x[:, H:H + HKV], x[:, H + HKV:])):
                for p in range(pos0 // page, (s.total[b] + page - 1) // page if n else 0):
                    lo, hi = max(p * page, pos0), min((p + 1) * page, s.total[b])
                    at, part = s.table[b, p], y[lo - pos0:hi - pos0]
                    mag = np.where(np.isfinite(part), np.abs(part), 0).max(axis=(0, 2)).astype(np.float32)
                    before = scale[at].copy() if lo > p * page else np.zeros(HKV, dtype=np.float32)
                    now = np.maximum(before, np.maximum(mag * (np.float32(1) / TOP[kind]), least))
                    for h in range(HKV):
                        if lo > p * page and now[h] > before[h]:
                            old = values(pool[at, h, :lo - p * page], kind).astype(np.float32)
                            pool[at, h, :lo - p * page] = to_codes(old * (before[h] / now[h]), kind)
                        with np.errstate(invalid="ignore"):
                            pool[at, h, lo - p * page:hi - p * page] = to_codes(part[:, h] * (np.float32(1) / now[h]), kind)
                        # in 64 bits: within half a step of the value (and the rounding of scale, reciprocal and product), where it is finite
                        exact, got = part[:, h].astype(np.float64), values(pool[at, h, lo - p * page:hi - p * page], kind) * now[h]
                        step = 0.5 * now[h] if kind == INT8 else np.maximum(np.abs(exact) / 16, now[h] * 2.0 ** -10)
                        ok = np.isfinite(exact)
                        assert np.all((np.abs(got - exact) <= step * 1.001 + np.abs(exact) * 2.0 ** -21)[ok])
                    scale[at] = now
        for name, pool, got, scale, got_s in zip("kv", pools, (s.pools[0][g], s.pools[1][g]), scales, (s.scales[0][g], s.scales[1][g])):
            assert np.array_equal(got_s.cpu().numpy(), scale), (name, "scale")
            got = got.cpu().numpy()
            # a negative number that rounds to nothing: the sign of the zero is the code's own
            same = (got == pool) | ((values(got, kind) == 0) & (values(pool, kind) == 0))
            assert same.all(), (name, g, np.argwhere(~same)[:4])
        got_q = q[g].float().cpu().numpy()
        cols = width if in_place else H * DH
        want = host[g].copy()[:, :cols] if in_place else want_q
        if in_place:
            want[:, :H * DH] = want_q
        want = bf16(want)
        assert np.array_equal(got_q[:, :cols], want, equal_nan=True)
        if not in_place and pad:
            assert (got_q[:, H * DH:] == 9.0).all()
        if spare:
            for two in s.pools:
                whole = two[g].as_strided((s.n_pages, spare), (HKV * page * DH + spare, 1), two[g].storage_offset() + HKV * page * DH)
                assert bool((whole == 0x7f).all())


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("rot,rot_dim", [(0, 0), (1, 128), (2, 128), (1, 32), (2, 48)])
def test_append_single_tokens(torch, ops, kind, page, rot, rot_dim):
    check_append(torch, ops, kind, 2, 6, 3, 128, page, [1] * 7, [1, page, page + 1, 2 * page, 2 * page - 1, 17, 300], rot, rot_dim, 1, one=True)


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("DH,rot,rot_dim", [(64, 1, 64), (64, 2, 32), (128, 1, 64), (64, 0, 0)])
def test_append_ragged_prompts(torch, ops, kind, page, DH, rot, rot_dim):
    check_append(torch, ops, kind, 1, 4, 2, DH, page, [1, 33, 0, 129, 2, 200, 15], [1, 40, 9, 129, 130, 263, 31], rot, rot_dim, 2)


def test_append_leaves_the_rest_alone(torch, ops):
    check_append(torch, ops, E4M3, 2, 2, 2, 64, 32, [3, 40, 1], [50, 70, 32], 1, 64, 3, spare=272, pad=24)
    check_append(torch, ops, INT8, 1, 3, 1, 64, 16, [5, 1], [20, 16], 2, 64, 4, in_place=True, pad=8)


@pytest.mark.parametrize("kind", [INT8, E4M3])
def test_append_of_what_is_no_number(torch, ops, kind):
    check_append(torch, ops, kind, 1, 2, 2, 64, 16, [30, 4], [37, 4], 0, 0, 5, poison=True)


def test_append_twice_is_append_once(torch, ops):
    check_append(torch, ops, E4M3, 1, 4, 4, 128, 64, [1, 70], [130, 90], 1, 128, 6, times=2)


def test_append_drops_what_has_no_place(torch, ops):
    """Tokens before position 0 and pages outside the pool: nothing is written, nothing else changes."""
    s = Setup(torch, ops, INT8, 1, 1, 64, 16, [4, 4], [2, 20], 7)
    table = s.table.copy()
    table[1, 1] = s.n_pages
    s.cache = ops.Cache(INT8, *s.pools, *s.scales, s.dev(table))
    x = s.bf16(s.n_tok, 3 * 64)[1]
    before = s.pools[0][0].cpu().numpy().copy()
    ops.hydra_op_cache_append(s.cache, s.lens, 1, 192, 0, [x], None, **s.call)
    after = s.pools[0][0].cpu().numpy()
    changed = np.argwhere((before != after).any(-1))
    assert {tuple(c) for c in changed} <= {(s.table[0, 0], 0, 0), (s.table[0, 0], 0, 1)} and len(changed) == 2


# ---- attention --------------------------------------------------------------------------------------------------------

def attention_64(s, g, q, H, causal, scale, total=None, lost=()):
    """(o, lse, sum p |v|, sum |q||k|) of every row and head; `lost`: (sequence, page) that the cache does not hold."""
    total = s.total if total is None else total
    o, lse = np.zeros((s.n_tok, H, s.DH)), np.full((s.n_tok, H), -np.inf)
    size, reach = np.zeros((s.n_tok, H, s.DH)), np.zeros((s.n_tok, H))
    for b in range(s.B):
        T = total[b]
        pages = s.table[b, :-(-T // s.page)]
        for h in range(s.HKV):
            if T == 0:
                continue
            k, v = ((values(p[g][pages, h], s.kind) * sc[g][pages, h].astype(np.float64)[:, None, None]).reshape(-1, s.DH)[:T]
                    for p, sc in ((s.k, s.ks), (s.v, s.vs)))
            there = np.array([(b, t // s.page) not in lost for t in range(T)])
            for j in range(s.new[b]):
                row, pos = s.ptr[b] + j, T - s.new[b] + j
                seen = there & (np.arange(T) <= pos) if causal else there
                if not seen.any():
                    continue
                for i in range(h * (H // s.HKV), (h + 1) * (H // s.HKV)):
                    x = q[row, i * s.DH:(i + 1) * s.DH].astype(np.float64)
                    z = (k[seen] @ x) * scale
                    m = z.max()
                    p = np.exp(z - m)
                    o[row, i], lse[row, i] = p @ v[seen] / p.sum(), m + np.log(p.sum())
                    size[row, i], reach[row, i] = p @ np.abs(v[seen]) / p.sum(), (np.abs(k[seen]) @ np.abs(x)).max() * scale
    return o, lse, size, reach


def check_attention(torch, ops, kind, G, H, HKV, DH, page, new, total, causal, seed, spare=0, one=False, pad=0, split=True, in_place=False, big=1.0,
                    s=None, lost=()):
    s = s or Setup(torch, ops, kind, G, HKV, DH, page, new, total, seed, spare, one)
    scale = 1.0 / math.sqrt(DH) / 3
    host, q = zip(*(s.bf16(s.n_tok, H * DH + pad, scale=big) for _ in range(G)))
    o = list(q) if in_place else [torch.full((s.n_tok, H * DH + pad), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(G)]
    lse = [torch.full((s.n_tok, H), 7.0, device="cuda") for _ in range(G)]
    which = {n: s.call[n] for n in ("n_tok", "max_q", "max_len")}
    size = ops.hydra_op_cache_attention_ws_bytes(s.cache, H, **which)
    ws = [torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(G)] if split and size else None
    again = [x.clone() for x in o]
    ops.hydra_op_cache_attention(s.cache, s.lens, H, H * DH + pad, H * DH + pad, causal, scale, list(q), o, lse, ws=ws, **s.call)
    if not in_place:
        ops.hydra_op_cache_attention(s.cache, s.lens, H, H * DH + pad, H * DH + pad, causal, scale, list(q), again, None, ws=ws, **s.call)
    torch.cuda.synchronize()
    for g in range(G):
        want, want_lse, mag, reach = attention_64(s, g, host[g], H, causal, scale, lost=lost)
        got = o[g].float().cpu().numpy()
        if not in_place:
            assert torch.equal(again[g], o[g])
            assert (got[:, H * DH:] == 7.0).all()
        got = got[:, :H * DH].reshape(s.n_tok, H, DH).astype(np.float64)
        # a score is off by its fp32 sum of DH products (2^-24 each and per addition at most) and the rounded scale: e; the weights by that and 2^-11
        # (rounding to f16 and hardware exp2); the result by bf16
        e = reach * (DH + 8) * 2.0 ** -24 + 2.0 ** -20
        assert np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + mag * (2.0 ** -10 + 2 * e[..., None]) + 1e-30), (g, np.abs(got - want).max())
        got_lse = lse[g].cpu().numpy().astype(np.float64)
        empty = np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), empty)
        assert np.all(got[empty] == 0)
        assert np.all((np.abs(got_lse - want_lse) <= 2 * e + 2.0 ** -20 * (8 + np.abs(want_lse)))[~empty])


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("DH", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attention_of_single_tokens(torch, ops, kind, DH, page):
    check_attention(torch, ops, kind, 2, 4, 2, DH, page, [1] * 8, [1, 15, 16, 17, 127, 128, 129, 500], True, 10, one=True)


@pytest.mark.parametrize("H,HKV", [(1, 1), (3, 3), (5, 1), (16, 1), (17, 1), (40, 2), (24, 8)])
def test_attention_of_shared_heads(torch, ops, H, HKV):
    check_attention(torch, ops, INT8, 1, H, HKV, 64, 32, [1, 2, 1], [77, 150, 3], True, 11)


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("DH,page", [(64, 16), (128, 64)])
def test_attention_of_ragged_calls(torch, ops, kind, causal, DH, page):
    """No token in a call, no token at all, a whole prompt, a prompt behind others, one token."""
    check_attention(torch, ops, kind, 1, 4, 2, DH, page, [0, 0, 130, 33, 1, 70], [0, 50, 130, 300, 257, 71], causal, 12)


@pytest.mark.parametrize("new,total", [([300], [300]), ([65, 1, 257], [1000, 1, 260]), ([128, 64], [129, 64])])
@pytest.mark.parametrize("kind,DH,page,H,HKV", [(INT8, 128, 64, 2, 2), (E4M3, 64, 16, 3, 1), (INT8, 64, 128, 5, 1), (E4M3, 128, 32, 4, 2)])
def test_attention_of_prompts(torch, ops, kind, DH, page, H, HKV, new, total):
    check_attention(torch, ops, kind, 1, H, HKV, DH, page, new, total, True, 13)


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("DH,page,H,HKV,new,total", [
    (128, 64, 12, 12, [200, 1, 131], [200, 40, 150]), (64, 128, 12, 12, [200, 1, 131], [200, 40, 150]),   # blocks of 128 rows
    (128, 16, 24, 6, [70, 65, 1], [700, 640, 130]), (128, 128, 32, 4, [40, 37, 0, 40], [400, 37, 5, 41]),  # of 256 rows, behind many keys
    (64, 16, 24, 6, [210, 65], [700, 640])])
def test_attention_of_prompts_by_blocks_of_rows(torch, ops, kind, causal, DH, page, H, HKV, new, total):
    """As many rows as the kernel for prompts takes: more than 256 tiles of 16."""
    check_attention(torch, ops, kind, 1, H, HKV, DH, page, new, total, causal, 23)


@pytest.mark.parametrize("kind,causal", [(INT8, True), (E4M3, True), (INT8, False)])
@pytest.mark.parametrize("DH,page", [(128, 16), (128, 64), (64, 32), (64, 128)])
def test_attention_of_more_than_1024_tiles(torch, ops, kind, causal, DH, page):
    check_attention(torch, ops, kind, 1, 32, 16, DH, page, [200, 1, 131], [230, 40, 131], causal, 25)


@pytest.mark.parametrize("kind,page", [(INT8, 64), (E4M3, 16)])
def test_attention_of_few_rows_behind_many_keys(torch, ops, kind, page):
    """Blocks of 256 rows, split runs of keys, joined."""
    check_attention(torch, ops, kind, 1, 4, 1, 128, page, [70], [38000], True, 26)


@pytest.mark.parametrize("DH,H", [(64, 1), (128, 1), (128, 4)])
def test_attention_of_prompts_behind_many_tokens(torch, ops, DH, H):
    """Few blocks of rows and many keys: split, and joined."""
    for page in (16, 64):
        check_attention(torch, ops, INT8, 1, H, 1, DH, page, [70, 66], [8300, 100], True, 24)


@pytest.mark.parametrize("one", [True, False])
def test_attention_of_long_sequences(torch, ops, one):
    check_attention(torch, ops, E4M3, 1, 2, 1, 64, 16, [1, 1] if one else [1, 3], [9000, 4097], True, 14, one=one)


def test_attention_with_and_without_scratch_and_in_place(torch, ops):
    for split in (True, False):
        check_attention(torch, ops, INT8, 2, 4, 4, 128, 64, [1, 1], [1500, 700], True, 15, split=split, pad=16, spare=256)
    check_attention(torch, ops, E4M3, 1, 4, 2, 128, 32, [1, 2], [150, 700], True, 16, in_place=True)
    check_attention(torch, ops, E4M3, 1, 4, 2, 128, 32, [150, 200], [150, 700], True, 16, in_place=True)


def test_attention_rows_before_the_first_token_see_nothing(torch, ops):
    for n in (4, 200):
        s = Setup(torch, ops, INT8, 1, 2, 64, 16, [n, n], [n // 2, n + 3], 17)
        check_attention(torch, ops, INT8, 1, 2, 2, 64, 16, None, None, True, 17, s=s)


@pytest.mark.parametrize("n", [2, 150])
@pytest.mark.parametrize("total", [400, 3000])
def test_rows_of_no_sequence_are_left_alone(torch, ops, n, total):
    """A call with room for more rows than q_ptr gives out (one captured for the most rows there may be): in one run of keys and in several."""
    s = Setup(torch, ops, INT8, 1, 2, 64, 32, [n, 1], [total, total // 2], 22)
    H, rows = 4, s.n_tok + 5
    q = torch.randn(rows, H * 64, device="cuda").to(torch.bfloat16)
    qkv = torch.randn(rows, (H + 4) * 64, device="cuda").to(torch.bfloat16)
    call = dict(s.call, n_tok=rows)
    which = {k: call[k] for k in ("n_tok", "max_q", "max_len")}
    size = ops.hydra_op_cache_attention_ws_bytes(s.cache, H, **which)
    assert (size > 0) == (total == 3000)
    ws = [torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")] if size else None
    o, lse = torch.full_like(q, 7.0), torch.full((rows, H), 7.0, device="cuda")
    ops.hydra_op_cache_attention(s.cache, s.lens, H, H * 64, H * 64, True, 0.125, [q], [o], [lse], ws=ws, **call)
    ops.hydra_op_cache_append(s.cache, s.lens, H, (H + 4) * 64, H * 64, [qkv], [q], **call)
    torch.cuda.synchronize()
    assert (o[s.n_tok:] == 7.0).all() and (lse[s.n_tok:] == 7.0).all()
    assert torch.isfinite(o[:s.n_tok]).all() and not (o[:s.n_tok] == 7.0).all(1).any()
    assert torch.equal(q[:s.n_tok], qkv[:s.n_tok, :H * 64]) and not torch.equal(q[s.n_tok:], qkv[s.n_tok:, :H * 64])


@pytest.mark.parametrize("n", [2, 150])
@pytest.mark.parametrize("kind", [INT8, E4M3])
def test_attention_of_pages_that_are_not_there(torch, ops, kind, n):
    s = Setup(torch, ops, kind, 1, 1, 64, 32, [n, n, n], [160, 300, 151], 18)
    for b, p, what in ((0, 0, -1), (1, 3, s.n_pages), (1, 4, 1 << 30)):
        s.table[b, p] = what
    s.cache = ops.Cache(kind, *s.pools, *s.scales, s.dev(s.table))
    s.table = np.clip(s.table, 0, s.n_pages - 1)
    check_attention(torch, ops, kind, 1, 2, 1, 64, 32, None, None, True, 18, s=s, lost={(0, 0), (1, 3), (1, 4)})


@pytest.mark.parametrize("n", [1, 140])
def test_attention_of_scales_far_apart(torch, ops, n):
    s = Setup(torch, ops, INT8, 1, 2, 128, 16, [n, n], [400, 333], 19)
    for scales, dev in zip((s.ks, s.vs), s.scales):
        scales[0][:] = 0.003 * (10.0 ** s.r.uniform(-12, 0, size=scales[0].shape)).astype(np.float32)
        scales[0][::5] = 2.0 ** -126
        dev[0].copy_(s.dev(scales[0]))
    check_attention(torch, ops, INT8, 1, 4, 2, 128, 16, None, None, True, 19, s=s, big=4.0)


def test_attention_of_rows_of_all_sizes(torch, ops):
    """Queries as small and as large as bf16 has them: the scores stay in proportion."""
    for n in (1, 130):
        for f in (2.0 ** -100, 2.0 ** 90):
            s = Setup(torch, ops, INT8, 1, 1, 64, 64, [n], [200], 20)
            x, q = s.bf16(s.n_tok, 64)
            got = []
            for by in (1.0, f):
                o, lse = torch.empty_like(q), torch.empty((s.n_tok, 1), device="cuda")
                ops.hydra_op_cache_attention(s.cache, s.lens, 1, 64, 64, True, 0.05 / by, [q * by], [o], [lse], **s.call)
                got.append((o.float(), lse))
            assert torch.equal(got[0][0], got[1][0]) or float((got[0][0] - got[1][0]).abs().max()) < 0.02 * float(got[0][0].abs().max())
            assert float((got[0][1] - got[1][1]).abs().max()) < 1e-4


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("n", [1, 150])
def test_a_cache_of_zeros(torch, ops, kind, n):
    """Scales of 2^-126 everywhere: the weights are those of equal scores, the result is zero."""
    s = Setup(torch, ops, kind, 1, 2, 64, 32, [n], [n], 22)
    x = torch.zeros((n, 6 * 64), dtype=torch.bfloat16, device="cuda")
    o, lse = torch.ones((n, 2 * 64), dtype=torch.bfloat16, device="cuda"), torch.empty((n, 2), device="cuda")
    ops.hydra_op_cache_append(s.cache, s.lens, 2, 384, 0, [x], None, **s.call)
    ops.hydra_op_cache_attention(s.cache, s.lens, 2, 384, 128, True, 0.1, [x], [o], [lse], **s.call)
    assert bool((o == 0).all())
    want = torch.log(torch.arange(1, n + 1, device="cuda").double())[:, None]
    assert float((lse.double() - want).abs().max()) < 2.0 ** -19


def test_offsets_past_32_bits(torch, ops):
    """Pages more than 4 GiB into a pool."""
    n_pages, hkv, page, dh = 40000, 8, 128, 128                                       # 5.2 GB each
    k, v = (torch.zeros((n_pages, hkv, page, dh), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.full((n_pages, hkv), 0.01, device="cuda") for _ in range(2))
    table = torch.tensor([[39999, 3]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([1], dtype=torch.int32, device="cuda")
    cache = ops.Cache(INT8, [k], [v], [ks], [vs], table)
    g = torch.Generator(device="cuda").manual_seed(1)
    for n, total in ((1, 1), (130, 131)):
        lens.fill_(total)
        ptr = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        x = torch.randn((n, 24 * dh), generator=g, device="cuda").to(torch.bfloat16)
        o = torch.empty((n, 8 * dh), dtype=torch.bfloat16, device="cuda")
        ops.hydra_op_cache_append(cache, lens, 8, 24 * dh, 0, [x], None, q_ptr=ptr, n_tok=n, max_q=n, max_len=256)
        ops.hydra_op_cache_attention(cache, lens, 8, 24 * dh, 8 * dh, True, 0.1, [x], [o], q_ptr=ptr, n_tok=n, max_q=n, max_len=256)
        if n == 1:                                                                       # one token seen: its value, to half a step
            want = x[:, 16 * dh:].float()
            assert bool(((o.float() - want).abs() <= want.abs().view(1, 8, dh).amax(-1).repeat_interleave(dh, 1) * (0.5 / 127 + 2.0 ** -8)).all())
    assert int((k[39999] != 0).sum()) > 0 and int((k[3, :, :3] != 0).sum()) > 0
    assert int((k[3, :, 3:] != 0).sum()) == 0 and int((k[:3] != 0).sum()) == 0
    assert bool(torch.isfinite(o.float()).all())


def test_decode_ops_on_a_stream_of_their_own_and_in_a_graph(torch, ops):
    s = Setup(torch, ops, E4M3, 1, 2, 128, 64, [1] * 4, [300, 65, 64, 129], 21, one=True)
    H, V = 4, 1000
    x = s.bf16(4, (H + 4) * 128)[1]
    q, o = torch.empty((4, H * 128), dtype=torch.bfloat16, device="cuda"), torch.empty((4, H * 128), dtype=torch.bfloat16, device="cuda")
    z, u = torch.randn((4, V), device="cuda"), torch.rand((4, V), device="cuda")
    t, k = torch.full((4,), 0.8, device="cuda"), torch.full((4,), 50, dtype=torch.int32, device="cuda")
    p, m = torch.full((4,), 0.9, device="cuda"), torch.zeros(4, device="cuda")
    token = torch.zeros(4, dtype=torch.int32, device="cuda")
    size = ops.hydra_op_cache_attention_ws_bytes(s.cache, H, max_len=300)
    ws = [torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")]
    cs = torch.rand((300, 128), device="cuda")

    def step():
        ops.hydra_op_cache_append(s.cache, s.lens, H, (H + 4) * 128, H * 128, [x], [q], rot=ops.ROT_HALVES, rot_dim=128, cos_sin=cs, max_len=300)
        ops.hydra_op_cache_attention(s.cache, s.lens, H, H * 128, H * 128, True, 0.088, [q], [o], ws=ws, max_len=300)
        ops.hydra_op_sample(ops.F32, 4, V, V, V, [z], [u], t, k, p, m, [token])

    step()
    torch.cuda.synchronize()
    want = o.clone(), token.clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(3):
        o.zero_(), token.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(token, want[1])
        (x.float() * 2).sum().item()


# ---- drawing tokens ---------------------------------------------------------------------------------------------------

def draw_64(z, u, t, k, p, m):
    """(token, logprob, how far the runner-up's score is behind, how near a kept set's edge any decision was)."""
    z = np.where(np.isnan(z), -np.inf, z.astype(np.float64))
    z = np.minimum(z, np.finfo(np.float32).max)
    if not (z > -np.inf).any():
        return -1, -np.inf, 1.0, 1.0
    zmax = z.max()
    lp = lambda i: z[i] - zmax - math.log(np.exp(z - zmax).sum())  # noqa: E731
    if not t > 0:
        i = int(np.argmax(z))
        return i, lp(i), 1.0, 1.0
    order = np.argsort(-z, kind="stable")
    order = order[z[order] > -np.inf]
    if k > 0:
        order = order[:k]
    w = np.exp((z[order] - zmax) / t)
    near = 1.0
    if p < 1:
        before = (np.cumsum(w) - w) / w.sum()
        near = np.abs(before - max(p, 0.0)).min()
        n = max(1, int((before < p).sum()))
        order, w = order[:n], w[:n]
    if m > 0:
        near = min(near, np.abs(w - min(m, 1)).min() if m < 1 else 1.0)
    order = order[w >= min(m, 1.0)]
    with np.errstate(divide="ignore"):
        s = np.maximum((z[order] - zmax) / t - np.log(-np.log(np.minimum(u[order].astype(np.float64), 1 - 2.0 ** -24))), -np.finfo(np.float32).max)
    best = np.lexsort((order, -s))
    gap = s[best[0]] - s[best[1]] if len(best) > 1 else 1.0
    return int(order[best[0]]), lp(order[best[0]]), gap, near


def check_sample(torch, ops, z, u, t, k, p, m, dtype="f32", pad=0):
    """z, u lists of [rows, V]."""
    rows, V = z[0].shape
    G = len(z)
    dev = lambda a, d: torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=d))).cuda()  # noqa: E731
    wide = [torch.full((rows, V + pad), 1e30, device="cuda") for _ in z]
    for a, b in zip(wide, z):
        a[:, :V] = dev(b, np.float32)
    if dtype == "bf16":
        wide = [a.to(torch.bfloat16) for a in wide]
        z = [a[:, :V].float().cpu().numpy() for a in wide]
    noise = [torch.full((rows, V + pad), 0.999, device="cuda") for _ in u]
    for a, b in zip(noise, u):
        a[:, :V] = dev(b, np.float32)
    token = [torch.full((rows,), -7, dtype=torch.int32, device="cuda") for _ in range(G)]
    logprob = [torch.full((rows,), 5.0, device="cuda") for _ in range(G)]
    ops.hydra_op_sample(ops.BF16 if dtype == "bf16" else ops.F32, rows, V, V + pad, V + pad, wide, noise, dev(t, np.float32), dev(k, np.int32), dev(p, np.float32),
                        dev(m, np.float32), token, logprob)
    torch.cuda.synchronize()
    told = 0
    for g in range(G):
        for r in range(rows):
            tok, lp, gap, near = draw_64(z[g][r], np.asarray(u[g][r], dtype=np.float32), t[r], k[r], np.float32(p[r]), np.float32(m[r]))
            got, got_lp = int(token[g][r]), float(logprob[g][r])
            # scores are off by a few units of 2^-24 times their size (30 at most where they can win), sums by 2^-23 or less
            if gap > 1e-4 and near > 2e-6:
                told += 1
                assert got == tok, (g, r, got, tok, t[r], k[r], p[r], m[r], gap, near)
                assert got_lp == lp or abs(got_lp - lp) <= 2.0 ** -19 * (4 + abs(lp)), (got_lp, lp)
    return told


def logits(r, rows, V, kind="ranked"):
    if kind == "flat":
        return r.normal(size=(rows, V)) * 0.01
    z = r.normal(size=(rows, V)) - 1.2 * np.log1p(r.permuted(np.tile(np.arange(V), (rows, 1)), axis=1))
    return z * (4.0 if kind == "peaked" else 1.0)


@pytest.mark.parametrize("V", [1, 2, 63, 1000, 8192, 8193, 30522, 32768, 32769, 70000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_filters(torch, ops, V, dtype):
    r = np.random.default_rng(V)
    rows, told = 16, 0
    z = [logits(r, rows, V, k).astype(np.float32) for k in ("ranked", "flat", "peaked")]
    u = [r.random((rows, V), dtype=np.float32) for _ in z]
    t = r.uniform(0.3, 1.5, rows)
    t[0] = 0.0
    k = np.where(r.random(rows) < 0.6, r.integers(1, 2 * V + 1, rows), 0)
    p = np.where(r.random(rows) < 0.6, r.uniform(0.0, 1.0, rows), 1.0)
    m = np.where(r.random(rows) < 0.3, r.uniform(0.0, 0.5, rows), 0.0)
    k[1], p[1], p[2] = 1, 0.5, 0.0
    told = check_sample(torch, ops, z, u, t, k, p, m, dtype, pad=V % 5)
    assert told >= 3 * rows * 0.8


@pytest.mark.parametrize("V", [5000, 32000, 100000, 150001, 262144])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("p", [1.0, 0.4, 0.9, 0.999])
def test_sample_keeps_few_and_many(torch, ops, V, dtype, p):
    """Kept sets of one token to tens of thousands: every way of finding the last one."""
    r = np.random.default_rng(V + int(1000 * p))
    ks = [0, 1, 2, 100, 128, 129, 257, 1000, 2048, 4096, 4097, 9000]
    z = logits(r, len(ks), V, "ranked").astype(np.float32)
    u = r.random((len(ks), V), dtype=np.float32)
    told = check_sample(torch, ops, [z, z * 0.01], [u, u], [0.9] * len(ks), ks, [p] * len(ks), [0.0] * len(ks), dtype)
    assert told >= len(ks)


@pytest.mark.parametrize("V", [90, 4097, 32003, 131072])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["any", "falling", "steps"])
def test_sample_cuts_that_hold_few_and_too_many(torch, ops, V, dtype, order):
    """min_p that leaves one token to nearly all, small top_k, both: logits in any order, falling with the index, and in steps of equal ones."""
    r = np.random.default_rng(V)
    rules = [(k, p, m) for k in (0, 1, 40, 96, 97, 3000) for p, m in ((1.0, 0.3), (0.95, 0.01), (0.97, 1e-4), (0.5, 1e-7), (0.9, 0.0))]
    k, p, m = (list(x) for x in zip(*rules))
    z = logits(r, len(rules), V, "ranked").astype(np.float32)
    if order != "any":
        z = -np.sort(-z, axis=1)
    if order == "steps":
        z = np.round(z * 2) / 2
    u = r.random((len(rules), V), dtype=np.float32)
    t = [1.3 if i % 2 else 0.8 for i in range(len(rules))]
    told = check_sample(torch, ops, [z, z * 0.05], [u, u], t, k, p, m, dtype, pad=V % 3)
    assert told >= len(rules)


@pytest.mark.parametrize("V", [500, 20000, 40000])
def test_sample_of_equal_logits(torch, ops, V):
    """Ties at the edge of the kept: the lower index stays."""
    r = np.random.default_rng(3)
    z = np.zeros((6, V), dtype=np.float32)
    z[1] = r.integers(-2, 2, V)
    z[2] = np.where(np.arange(V) % 7 == 3, 1e-45, 0.0)
    z[3, V // 2] = 5.0
    z[4] = r.integers(0, 2, V) * 3e38
    z[5] = np.where(r.random(V) < 0.5, -3e38, np.where(r.random(V) < 0.5, 3e38, 0))
    u = r.random((6, V), dtype=np.float32)
    for k in (1, 5, 300, V // 2):
        told = check_sample(torch, ops, [z], [u], [1.0] * 6, [k] * 6, [1.0] * 6, [0.0] * 6)
        assert told >= 5
    # the exact share of equal tokens: k of them, half of those
    check_sample(torch, ops, [z[:1]], [u[:1]], [0.7], [V // 5 * 2 + 1], [0.5], [0.0])


def test_sample_of_what_is_no_number(torch, ops):
    V = 3000
    r = np.random.default_rng(4)
    z = r.normal(size=(8, V)).astype(np.float32)
    u = r.random((8, V), dtype=np.float32)
    z[0, :] = -np.inf
    z[1, :] = np.nan
    z[2, 5:] = -np.inf
    z[3, ::2] = np.nan
    z[4, 77], z[4, 99] = np.inf, np.inf
    z[5, :] = -3.4e38
    z[5, 9] = -1.0
    u[6, :] = 0.0
    u[7, 1000] = 1.0
    for k, p, m, t in ((0, 1.0, 0.0, 1.0), (10, 1.0, 0.0, 0.7), (0, 0.9, 0.0, 1.2), (50, 0.8, 0.05, 1.0), (0, 1.0, 0.0, 0.0), (0, 1.0, 2.0, 1.0)):
        check_sample(torch, ops, [z], [u], [t] * 8, [k] * 8, [p] * 8, [m] * 8)
    check_sample(torch, ops, [z[:1]], [u[:1]], [float("nan")], [3], [0.5], [0.0])


def test_sample_frequencies(torch, ops):
    """Draws over many uniforms come with the probabilities of the kept: each frequency within 5 standard deviations."""
    V, n = 11, 40000
    r = np.random.default_rng(5)
    z = np.tile(r.normal(size=V).astype(np.float32), (n, 1))
    u = torch.rand((n, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    token = torch.empty(n, dtype=torch.int32, device="cuda")
    full = lambda v, d: torch.full((n,), v, dtype=d, device="cuda")  # noqa: E731
    ops.hydra_op_sample(ops.F32, n, V, V, V, [torch.from_numpy(z).cuda()], [u], full(0.9, torch.float32), full(8, torch.int32), full(0.95, torch.float32),
                        full(0.0, torch.float32), [token])
    got = np.bincount(token.cpu().numpy(), minlength=V) / n
    order = np.argsort(-z[0], kind="stable")[:8]
    w = np.exp(z[0][order] / 0.9)
    keep = order[:int((np.cumsum(w) - w < 0.95 * w.sum()).sum())]
    want = np.zeros(V)
    want[keep] = np.exp(z[0][keep] / 0.9) / np.exp(z[0][keep] / 0.9).sum()
    assert np.all(np.abs(got - want) <= 5 * np.sqrt(want * (1 - want) / n)), (got, want)


# ---- cases of their own -----------------------------------------------------------------------------------------------

BF16_TOP = float.fromhex("0x1.fep127")


@pytest.mark.parametrize("V", [301, 3000, 70000])
@pytest.mark.parametrize("k,p,m,t", [(0, 1.0, 0.0, 0.0), (0, 1.0, 0.05, 1.0), (0, 1.0, 0.0, 1.0), (10, 1.0, 0.0, 0.7), (200, 1.0, 0.0, 0.7), (200, 0.9, 0.0, 0.7),
                                     (0, 0.9, 0.0, 1.2), (50, 0.8, 0.05, 1.0), (0, 0.9, 0.05, 1.0)], ids=str)
def test_sample_of_16_bit_logits_that_are_no_numbers(torch, ops, V, k, p, m, t):
    """+inf counts as the largest bf16 number in every form: alone, twice, and beside that number itself; NaN and -inf are never drawn."""
    r = np.random.default_rng(V)
    z = r.normal(size=(6, V)).astype(np.float32)
    u = r.random((6, V), dtype=np.float32)
    z[0, 77] = np.inf
    z[1, 77], z[1, 99] = np.inf, np.inf
    z[2, 20], z[2, 250] = np.inf, BF16_TOP
    z[3, ::2], z[3, 101] = np.nan, np.inf
    z[4, :], z[4, 9] = -np.inf, np.inf
    z[5, ::3] = np.nan
    z_dev = torch.from_numpy(z).cuda().to(torch.bfloat16)
    full = lambda v, d: torch.full((6,), v, dtype=d, device="cuda")  # noqa: E731
    token, logprob = full(-7, torch.int32), full(5.0, torch.float32)
    ops.hydra_op_sample(ops.BF16, 6, V, V, V, [z_dev], [torch.from_numpy(u).cuda()], full(t, torch.float32), full(k, torch.int32), full(p, torch.float32),
                        full(m, torch.float32), [token], [logprob])
    got, got_lp = token.cpu().numpy(), logprob.cpu().numpy()
    assert ((got >= 0) & (got < V)).all(), got
    held = np.minimum(z_dev.float().cpu().numpy(), BF16_TOP)
    for i in range(6):
        tok, lp, gap, near = draw_64(held[i], u[i], t, k, np.float32(p), np.float32(m))
        assert gap > 1e-4 and near > 2e-6 or i == 5                     # ordinary logits may be close; these are not
        if gap > 1e-4 and near > 2e-6:
            assert got[i] == tok and abs(got_lp[i] - lp) <= 2.0 ** -19 * (4 + abs(lp)), (i, got[i], tok, got_lp[i], lp)


@pytest.mark.parametrize("total", [400, 3000])
def test_rows_past_the_most_of_a_sequence_are_left_alone(torch, ops, total):
    """A sequence with more rows in q_ptr than max_q allows: its first max_q rows are answered, the others left alone, in one run of keys and in several."""
    s = Setup(torch, ops, INT8, 1, 2, 64, 32, [6, 0, 2, 70], [total, total // 2, total, total], 27)
    H, most = 4, 3
    q = torch.randn(s.n_tok, H * 64, device="cuda").to(torch.bfloat16)
    call = dict(s.call, max_q=most)
    size = ops.hydra_op_cache_attention_ws_bytes(s.cache, H, **{k: call[k] for k in ("n_tok", "max_q", "max_len")})
    assert (size > 0) == (total == 3000)
    ws = [torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")] if size else None
    o, lse = torch.full_like(q, 7.0), torch.full((s.n_tok, H), 7.0, device="cuda")
    ops.hydra_op_cache_attention(s.cache, s.lens, H, H * 64, H * 64, True, 0.125, [q], [o], [lse], ws=ws, **call)
    answered = torch.tensor([i for b, n in enumerate(s.new) for i in range(s.ptr[b], s.ptr[b] + min(n, most))], device="cuda")
    rest = torch.ones(s.n_tok, dtype=torch.bool, device="cuda")
    rest[answered] = False
    assert (o[rest] == 7.0).all() and (lse[rest] == 7.0).all()
    assert torch.isfinite(o[answered]).all() and not (o[answered] == 7.0).all(1).any()


def attention_64_by_heads(s, g, q, H, causal, scale, lost=(), most=False):
    """attention_64 for larger calls: the same in products of all rows of a key/value head.  most: and the row's largest weight times its page's scale of
    values."""
    o, lse = np.zeros((s.n_tok, H, s.DH)), np.full((s.n_tok, H), -np.inf)
    size, reach, largest = np.zeros((s.n_tok, H, s.DH)), np.zeros((s.n_tok, H)), np.zeros((s.n_tok, H))
    share = H // s.HKV
    for b in range(s.B):
        T, n = s.total[b], s.new[b]
        if not T or not n:
            continue
        pages = s.table[b, :-(-T // s.page)]
        there = np.array([(b, t // s.page) not in lost for t in range(T)])
        seen = np.repeat(there & ((np.arange(T) <= T - n + np.arange(n)[:, None]) if causal else np.ones((n, 1), dtype=bool)), share, axis=0)
        some = seen.any(1)
        for h in range(s.HKV):
            k, v = ((values(p[g][pages, h], s.kind) * sc[g][pages, h].astype(np.float64)[:, None, None]).reshape(-1, s.DH)[:T]
                    for p, sc in ((s.k, s.ks), (s.v, s.vs)))
            k, v = np.where(there[:, None], k, 0), np.where(there[:, None], v, 0)
            at = np.s_[s.ptr[b]:s.ptr[b + 1], h * share:(h + 1) * share]
            x = q[s.ptr[b]:s.ptr[b + 1]].astype(np.float64).reshape(n, H, s.DH)[:, h * share:(h + 1) * share].reshape(-1, s.DH)
            z = np.where(seen, x @ k.T * scale, -np.inf)
            m = np.where(some, z.max(1), 0)
            p = np.exp(z - m[:, None])
            total = np.where(some, p.sum(1), 1)
            far = np.where(seen, np.abs(x) @ np.abs(k).T, 0).max(1) * scale
            with np.errstate(divide="ignore"):
                lse[at] = np.where(some, m + np.log(total), -np.inf).reshape(n, share)
            o[at], size[at] = (p @ v / total[:, None]).reshape(n, share, -1), (p @ np.abs(v) / total[:, None]).reshape(n, share, -1)
            reach[at] = far.reshape(n, share)
            if most:
                largest[at] = ((p * np.repeat(s.vs[g][pages, h].astype(np.float64), s.page)[:T]).max(1) / total).reshape(n, share)
    return (o, lse, size, reach, largest) if most else (o, lse, size, reach)


def check_rows_of_one_page_each(torch, ops, kind, DH, page, H, HKV, new, total, step, order, ws=True, slots=5):
    """Every row has all its weight on the pages of one slot (page number modulo `slots`), whose values are 2^-(step * slot) of the largest: the result is as
    near to that slot's values as its own size asks, however small they are.  order "grows": the small ones first, over the whole sequence."""
    s = Setup(torch, ops, kind, 1, HKV, DH, page, new, total, 31)
    r = np.random.default_rng(32)
    few = {INT8: 3, E4M3: 8}[kind]                                      # of 127 or 448: what a key has in the other columns
    for b in range(s.B):
        n = -(-total[b] // page)
        for i in range(n):
            slot = i % slots if order == "any" else (n - 1 - i) * slots // n
            at = s.table[b, i]
            x = r.integers(-few, few + 1, size=(HKV, page, DH)).astype(np.float32)
            x[..., slot] = TOP[kind]
            s.k[0][at] = to_codes(x, kind)
            s.v[0][at] = to_codes((r.normal(size=(HKV, page, DH)) * TOP[kind] / 3).astype(np.float32), kind)
            s.ks[0][at] = np.float32(1) / TOP[kind]
            s.vs[0][at] = np.float32(0.01 * 2.0 ** (-step * slot)) * r.uniform(0.7, 1.4, HKV).astype(np.float32)
    for pools, scales, k, sc in ((s.pools[0], s.scales[0], s.k, s.ks), (s.pools[1], s.scales[1], s.v, s.vs)):
        pools[0].copy_(s.dev(k[0]))
        scales[0].copy_(s.dev(sc[0]))
    x = r.normal(size=(s.n_tok, H, DH)) * 0.05
    row = np.arange(s.n_tok)[:, None] + np.arange(H)[None]
    np.put_along_axis(x, (row % slots)[..., None], 40.0, axis=-1)
    q = bf16(x.reshape(s.n_tok, -1))
    which = {n: s.call[n] for n in ("n_tok", "max_q", "max_len")}
    size = ops.hydra_op_cache_attention_ws_bytes(s.cache, H, **which) if ws else 0
    scratch = [torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")] if size else None
    o, lse = torch.full((s.n_tok, H * DH), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((s.n_tok, H), 7.0, device="cuda")
    ops.hydra_op_cache_attention(s.cache, s.lens, H, H * DH, H * DH, False, 1.0, [s.dev(q).to(torch.bfloat16)], [o], [lse], ws=scratch, **s.call)
    want, want_lse, mag, reach = attention_64_by_heads(s, 0, q, H, False, 1.0)
    got, got_lse = o.float().cpu().numpy().reshape(s.n_tok, H, DH).astype(np.float64), lse.cpu().numpy().astype(np.float64)
    e = reach * (DH + 8) * 2.0 ** -24 + 2.0 ** -20                      # as in check_attention
    off = np.abs(got - want) / (2.0 ** -8 * np.abs(want) + mag * (2.0 ** -10 + 2 * e[..., None]) + 1e-30)
    assert off.max() <= 1, (off.max(), [float(off[row % slots == i].max()) for i in range(slots)])
    assert np.all(np.abs(got_lse - want_lse) <= 2 * e + 2.0 ** -20 * (8 + np.abs(want_lse)))


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("order", ["any", "grows"])
@pytest.mark.parametrize("step", [5, 10, 15])
@pytest.mark.parametrize("DH,page,total", [(64, 16, 400), (128, 64, 330), (128, 16, 1500)])
def test_attention_of_tokens_that_see_small_values_alone(torch, ops, kind, order, step, DH, page, total):
    check_rows_of_one_page_each(torch, ops, kind, DH, page, 10, 2, [1, 3], [total, total - 7], step, order)


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("order", ["any", "grows"])
@pytest.mark.parametrize("step", [5, 10, 15])
@pytest.mark.parametrize("DH,page", [(64, 16), (128, 64)])
def test_attention_of_prompts_that_see_small_values_alone(torch, ops, kind, order, step, DH, page):
    check_rows_of_one_page_each(torch, ops, kind, DH, page, 60, 12, [150, 100], [330, 320], step, order)


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("order", ["any", "grows"])
@pytest.mark.parametrize("step", [5, 10, 15])
def test_attention_of_small_values_alone_in_one_run_of_many_pages(torch, ops, kind, order, step):
    """Without scratch a run is all of a sequence: more pages than the kernels know at a time (64; 512 for prompts), the largest values among the last."""
    check_rows_of_one_page_each(torch, ops, kind, 128, 16, 10, 2, [2, 1], [3000, 1900], step, order, ws=False)
    check_rows_of_one_page_each(torch, ops, kind, 64, 16, 60, 12, [20], [18000], step, order, ws=False)


# ---- the kernel for prompts, in every form ----------------------------------------------------------------------------


def check_prompts(torch, ops, s, H, causal, rows, split, ws=True, in_place=False, pad=0, lost=(), scale=0.05, n_tok=None):
    """A call that the kernel for prompts takes with `rows` rows to a workgroup, in several runs of keys or one, against 64 bits.  Tolerances: those of
    check_attention, and what f16 has below its normal numbers.  Weights are held as w_t = 2^7 p_t v_t / (at most the largest p v of the row), p the weight, v the
    page's scale of values; below 2^-14 f16 rounds them to 2^-25, so that T keys of codes up to the kind's largest are off by T 2^-32 times that code times the
    row's largest p v.  It tells in columns alone in which the keys that the row looks at have the code 0."""
    n_tok = n_tok or s.n_tok
    call = dict(s.call, n_tok=n_tok)
    which = {n: call[n] for n in ("n_tok", "max_q", "max_len")}
    plan = ops.hydra_op_cache_attention_plan(s.cache, H, **which)
    assert plan[:2] == (rows, rows // 32), plan
    size = ops.hydra_op_cache_attention_ws_bytes(s.cache, H, **which) if ws else 0
    assert ((plan[2] > 1) if ws else False) == (size > 0) == split, (plan, size)
    scratch = [torch.full((size,), 0xff, dtype=torch.uint8, device="cuda") for _ in range(s.G)] if size else None
    host, q = zip(*(s.bf16(n_tok, H * s.DH + pad) for _ in range(s.G)))
    q = [x.clone() for x in q]
    o = q if in_place else [torch.full((n_tok, H * s.DH + pad), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(s.G)]
    lse = [torch.full((n_tok, H), 7.0, device="cuda") for _ in range(s.G)]
    ops.hydra_op_cache_attention(s.cache, s.lens, H, H * s.DH + pad, H * s.DH + pad, causal, scale, q, o, lse, ws=scratch, **call)
    torch.cuda.synchronize()
    for g in range(s.G):
        want, want_lse, mag, reach, most = attention_64_by_heads(s, g, host[g][:s.n_tok, :H * s.DH], H, causal, scale, lost=lost, most=True)
        least = max(s.total) * 2.0 ** -32 * float(TOP[s.kind]) * most[..., None]
        got = o[g].float().cpu().numpy()
        assert in_place or (got[s.n_tok:] == 7.0).all() and (got[:, H * s.DH:] == 7.0).all() and bool((lse[g][s.n_tok:] == 7.0).all())
        got = got[:s.n_tok, :H * s.DH].reshape(s.n_tok, H, s.DH).astype(np.float64)
        e = reach * (s.DH + 8) * 2.0 ** -24 + 2.0 ** -20
        off = np.abs(got - want) / (2.0 ** -8 * np.abs(want) + mag * (2.0 ** -10 + 2 * e[..., None]) + least + 1e-30)
        assert off.max() <= 1, (g, off.max(), np.unravel_index(off.argmax(), off.shape))
        got_lse, empty = lse[g][:s.n_tok].cpu().numpy().astype(np.float64), np.isneginf(want_lse)
        assert np.array_equal(np.isneginf(got_lse), empty) and np.all(got[empty] == 0)
        assert np.all((np.abs(got_lse[~empty] - want_lse[~empty]) <= (2 * e + 2.0 ** -20 * (8 + np.abs(want_lse)))[~empty]))


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("DH,page", [(128, 64), (128, 16), (64, 32), (64, 128)])
def test_prompts_of_a_group(torch, ops, kind, causal, DH, page):
    """Three models, four waves, one run; sequences without tokens in the call, and without any."""
    s = Setup(torch, ops, kind, 3, 8, DH, page, [200, 0, 131, 0, 77], [230, 50, 131, 0, 300], 41, spare=64)
    check_prompts(torch, ops, s, 16, causal, 128, False, pad=8)


@pytest.mark.parametrize("kind,DH,page,causal", [(INT8, 128, 64, True), (E4M3, 128, 16, True), (E4M3, 64, 64, False), (INT8, 64, 16, True)])
def test_prompts_in_several_runs(torch, ops, kind, DH, page, causal):
    """Four waves, few blocks of rows behind many keys, two models: joined; the second sequence ends inside the first run."""
    s = Setup(torch, ops, kind, 2, 2, DH, page, [500, 130], [3000, 133], 42)
    check_prompts(torch, ops, s, 2, causal, 128, True)
    check_prompts(torch, ops, s, 2, causal, 128, False, ws=False)
    check_prompts(torch, ops, s, 2, causal, 128, True, n_tok=s.n_tok + 3)     # rows of no sequence


@pytest.mark.parametrize("kind,page,causal", [(INT8, 64, True), (E4M3, 64, False), (E4M3, 16, True), (INT8, 32, False)])
def test_prompts_by_eight_waves(torch, ops, kind, page, causal):
    """Blocks of 256 rows: few rows behind many keys, two models, in one run (without scratch) and in several."""
    s = Setup(torch, ops, kind, 2, 4, 128, page, [40, 33, 0, 7], [1500, 1411, 20, 1300], 43)
    check_prompts(torch, ops, s, 36, causal, 256, True)
    check_prompts(torch, ops, s, 36, causal, 256, False, ws=False)


@pytest.mark.parametrize("kind,causal", [(INT8, True), (E4M3, False)])
@pytest.mark.parametrize("H,rows", [(132, 128), (528, 256)])
def test_prompts_over_more_pages_than_are_known_at_a_time(torch, ops, kind, causal, H, rows):
    """A run of more than 512 pages of 16 tokens (without scratch), and the largest values among the last."""
    s = Setup(torch, ops, kind, 2, 2, 128, 16, [1, 1, 1, 1], [20000, 8193, 8192, 16390], 44)
    for g in range(2):
        for b in range(4):
            s.vs[g][s.table[b, 512:-(-s.total[b] // 16)]] *= 300.0
        s.scales[1][g].copy_(s.dev(s.vs[g]))
    check_prompts(torch, ops, s, H, causal, rows, False, ws=False)
    check_prompts(torch, ops, s, H, causal, rows, True)


@pytest.mark.parametrize("kind", [INT8, E4M3])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("split", [True, False])
def test_prompts_with_pages_that_are_not_there(torch, ops, kind, page, split):
    s = Setup(torch, ops, kind, 1, 12, 128, page, [150, 150, 100], [1100, 300, 151], 45)
    lost = {(0, 0), (1, 1), (0, 1000 // page), (2, 0)} | ({(0, 40), (0, 41), (0, 42), (0, 43), (1, 5)} if page == 16 else set())
    for n, (b, p) in enumerate(sorted(lost)):
        s.table[b, p] = (-1, s.n_pages, 1 << 30)[n % 3]
    s.cache = ops.Cache(kind, *s.pools, *s.scales, s.dev(s.table))
    s.table = np.clip(s.table, 0, s.n_pages - 1)
    check_prompts(torch, ops, s, 60, True, 128, split, ws=split, lost=lost)


@pytest.mark.parametrize("kind,DH", [(INT8, 128), (E4M3, 64)])
def test_prompts_in_place_and_rows_that_see_nothing(torch, ops, kind, DH):
    s = Setup(torch, ops, kind, 2, 8, DH, 32, [190, 200, 150], [95, 203, 150], 46)     # the first one's first 95 rows lie before its first token
    check_prompts(torch, ops, s, 24, True, 128, False, in_place=True)
    check_prompts(torch, ops, s, 24, True, 128, False, pad=16)
    s = Setup(torch, ops, kind, 1, 3, DH, 64, [300, 20], [2300, 10], 47)
    check_prompts(torch, ops, s, 15, True, 128, True, in_place=True)


def test_prompts_with_more_rows_than_a_sequence_may_have(torch, ops):
    for total, split in ((400, False), (3000, True)):
        s = Setup(torch, ops, INT8, 1, 8 if split else 24, 64, 32, [160, 0, 200], [total, 30, total], 48)
        H, most, n = 4 * s.HKV, 150, s.n_tok
        call = dict(s.call, max_q=most)
        which = {k: call[k] for k in ("n_tok", "max_q", "max_len")}
        plan = ops.hydra_op_cache_attention_plan(s.cache, H, **which)
        assert plan[0] == 128 and (plan[2] > 1) == split, plan
        ws = [torch.full((ops.hydra_op_cache_attention_ws_bytes(s.cache, H, **which),), 0xff, dtype=torch.uint8, device="cuda")] if split else None
        q = torch.randn(n, H * 64, device="cuda").to(torch.bfloat16)
        o = torch.full_like(q, 7.0)
        ops.hydra_op_cache_attention(s.cache, s.lens, H, H * 64, H * 64, True, 0.125, [q], [o], ws=ws, **call)
        assert (o[150:160] == 7.0).all() and (o[310:] == 7.0).all()
        for part in (o[:150], o[160:310]):
            assert torch.isfinite(part).all() and not (part == 7.0).all(1).any()


@pytest.mark.parametrize("kind", [INT8, E4M3])
def test_prompts_over_a_cache_of_zeros_and_queries_of_all_sizes(torch, ops, kind):
    s = Setup(torch, ops, kind, 1, 8, 64, 32, [300, 290], [300, 290], 49)
    H, n = 32, s.n_tok
    assert ops.hydra_op_cache_attention_plan(s.cache, H, **{k: s.call[k] for k in ("n_tok", "max_q", "max_len")})[0] == 128
    x, q = s.bf16(n, H * 64)
    got = []
    for by in (1.0, 2.0 ** -100, 2.0 ** 90):
        o, lse = torch.empty_like(q), torch.empty((n, H), device="cuda")
        ops.hydra_op_cache_attention(s.cache, s.lens, H, H * 64, H * 64, True, 0.05 / by, [q * by], [o], [lse], **s.call)
        got.append((o.float(), lse))
    for o, lse in got[1:]:
        assert float((o - got[0][0]).abs().max()) < 0.02 * float(got[0][0].abs().max()) and float((lse - got[0][1]).abs().max()) < 1e-4
    zeros = torch.zeros((n, (H + 16) * 64), dtype=torch.bfloat16, device="cuda")
    o, lse = torch.ones((n, H * 64), dtype=torch.bfloat16, device="cuda"), torch.empty((n, H), device="cuda")
    ops.hydra_op_cache_append(s.cache, s.lens, H, (H + 16) * 64, 0, [zeros], None, **s.call)
    ops.hydra_op_cache_attention(s.cache, s.lens, H, (H + 16) * 64, H * 64, True, 0.1, [zeros], [o], [lse], **s.call)
    want = torch.log(torch.cat([torch.arange(1, m + 1, device="cuda") for m in s.new]).double())[:, None]
    assert bool((o == 0).all()) and float((lse.double() - want).abs().max()) < 2.0 ** -19


@pytest.mark.parametrize("n,total,rows", [(170, 1300, 128), (140, 1300, 256)])
def test_prompts_over_pages_past_32_bits(torch, ops, n, total, rows):
    """Pages more than 4 GiB into a pool of 5.2 GB."""
    s = Setup(torch, ops, INT8, 1, 8, 128, 128, [n], [total], 50)
    at = np.array([39999, 3, 39000, 35001, 2, 37777, 33000, 39998, 0, 36000, 34567])
    pools = [[torch.zeros((40000, 8, 128, 128), dtype=torch.int8, device="cuda")] for _ in range(2)]
    scales = [[torch.full((40000, 8), 0.01, device="cuda")] for _ in range(2)]
    there = torch.from_numpy(at).cuda()
    for pool, scale, host, sc in zip(pools, scales, (s.k, s.v), (s.ks, s.vs)):
        pool[0][there] = s.dev(host[0][s.table[0]].view(np.int8))
        scale[0][there] = s.dev(sc[0][s.table[0]])
    s.cache = ops.Cache(INT8, *pools, *scales, s.dev(at[None].astype(np.int32)))
    check_prompts(torch, ops, s, 64, True, rows, True)
    check_prompts(torch, ops, s, 64, True, rows, False, ws=False)
