"""What the serving operators refuse, before anything is launched (no GPU): the status, the text and that the size query agrees."""
import ctypes as C

import pytest

from paper_2107_06469_amd import ops
from paper_2107_06469_amd.hydra import lib

A = 1 << 20                       # an address that is never looked at, well aligned


def cache(G=1, table=True, **kw):
    d = dict(kind=0, B=3, HKV=2, DH=128, page=64, n_pages=10, max_pages=4, G=G, n_tok=3, max_q=1, max_len=256, page_bytes=0, page_table=A, lens=A, q_ptr=0)
    d.update(kw)
    tabs = [(C.c_void_p * 16)(*[d.pop(n, A)] * 16) for n in ("k", "v", "k_scale", "v_scale")]
    return (*d.values(), *[C.addressof(t) if table else 0 for t in tabs]), tabs


def pointers(at=A):
    return (C.c_void_p * 16)(*[at] * 16)


def append(H=4, ld_qkv=1024, ld_q=512, rot=0, rot_dim=0, cs=A, qkv=A, q=A, **kw):
    d, keep = cache(**kw)
    tabs = pointers(qkv), pointers(q if q is not None else A)
    st = ops._L().hydra_op_cache_append(ops._append_desc(*d, H, ld_qkv, ld_q, rot, rot_dim, cs or 0, *[C.addressof(t) for t in tabs]), None)
    return st, lib().hydra_ops_last_error().decode()


def attend(H=4, ld_q=512, ld_o=512, scale=0.1, q=A, o=A, lse=A, ws=None, **kw):
    d, keep = cache(**kw)
    tabs = pointers(q), pointers(o), pointers(lse), pointers(ws or A)
    at = [C.addressof(t) for t in tabs]
    if not ws:
        at[3] = 0
    st = ops._L().hydra_op_cache_attention(ops._attention_desc(*d, H, ld_q, ld_o, 1, scale, *at, 0), None)
    return st, lib().hydra_ops_last_error().decode()


CACHE = [dict(kind=2), dict(kind=-1), dict(DH=96), dict(DH=0), dict(page=8), dict(page=48), dict(page=256), dict(B=0), dict(B=70000), dict(HKV=0),
         dict(n_pages=0), dict(max_pages=0), dict(max_len=0), dict(max_len=257), dict(n_tok=0), dict(max_q=0), dict(max_q=2), dict(n_tok=4),
         dict(page_bytes=64 * 256 - 16), dict(page_bytes=64 * 256 + 8), dict(page_table=0), dict(lens=0), dict(k=0), dict(v=0), dict(k_scale=0),
         dict(v_scale=0), dict(k=A + 8), dict(v=A + 1), dict(G=0), dict(G=17), dict(table=False), dict(H=0), dict(H=3), dict(H=-2),
         dict(max_q=5, n_tok=4, q_ptr=A)]


@pytest.mark.parametrize("bad", CACHE + [dict(ld_qkv=1016), dict(ld_qkv=1028), dict(ld_q=504), dict(ld_q=516), dict(qkv=0), dict(qkv=A + 2), dict(q=0),
                                         dict(q=A + 8), dict(rot=3, rot_dim=64), dict(rot=1, rot_dim=0), dict(rot=1, rot_dim=136),
                                         dict(rot=2, rot_dim=24), dict(rot=1, rot_dim=64, cs=None)], ids=str)
def test_append_refuses(bad):
    st, why = append(**bad)
    assert st == 1 and why.startswith("hydra_op_cache_append: "), (st, why)


@pytest.mark.parametrize("bad", CACHE + [dict(ld_q=504), dict(ld_o=508), dict(ld_o=256), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                         dict(scale=float("inf")), dict(q=0), dict(o=0), dict(q=A + 2), dict(o=A + 4), dict(ws=A + 4)], ids=str)
def test_attention_refuses(bad):
    st, why = attend(**bad)
    assert st == 1 and why.startswith("hydra_op_cache_attention: "), (st, why)


def test_attention_scratch_sizes():
    """0 for what is refused and for short sequences; the same for any number of calls; growing with the sequences."""
    size = lambda H=4, **kw: ops._L().hydra_op_cache_attention_ws_bytes(ops._cache_desc(*cache(**kw)[0]), H)  # noqa: E731
    assert size(kind=5) == 0 and size(H=3) == 0 and size(max_len=100) == 0
    long = dict(max_pages=1000, max_len=64000)
    assert size(**long) == size(**long) > 0
    assert size(**long) % 4 == 0


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(rows=0), dict(V=0), dict(V=(1 << 24) + 1, ldz=1 << 25, ldu=1 << 25), dict(ldz=99), dict(ldu=99), dict(G=0), dict(G=17),
                                 dict(logits=0), dict(u=0), dict(token=0), dict(logprob=0), dict(t=None), dict(k=None), dict(p=None), dict(m=None)], ids=str)
def test_sample_refuses(bad):
    a = dict(dtype=0, rows=4, V=100, ldz=100, ldu=100, G=1, logits=A, u=A, t=A, k=A, p=A, m=A, token=A, logprob=A)
    a.update(bad)
    st = ops._L().hydra_op_sample(a["dtype"], a["rows"], a["V"], a["ldz"], a["ldu"], a["G"], pointers(a["logits"]), pointers(a["u"]), a["t"], a["k"], a["p"],
                                  a["m"], pointers(a["token"]), pointers(a["logprob"]), None)
    assert st == 1 and lib().hydra_ops_last_error().decode().startswith("hydra_op_sample: ")


def test_descriptors_are_laid_out_as_declared():
    """Sizes of the packed records against the C structures."""
    ints, ptr = C.c_int, C.c_void_p
    cache_fields = [(f"i{n}", ints) for n in range(11)] + [("page_bytes", C.c_size_t)] + [(f"p{n}", ptr) for n in range(7)]
    desc = type("D", (C.Structure,), {"_fields_": cache_fields})
    more = {ops._cache_desc: [], ops._append_desc: [(f"j{n}", ints) for n in range(5)] + [(f"q{n}", ptr) for n in range(3)],
            ops._attention_desc: [(f"j{n}", ints) for n in range(4)] + [("scale", C.c_float)] + [(f"q{n}", ptr) for n in range(4)] + [("ws_bytes", C.c_size_t)]}
    for pack, rest in more.items():
        whole = type("W", (C.Structure,), {"_fields_": [("cache", desc)] + rest})
        values = [1] * 11 + [2] + [3] * 7 + [0.5 if t is C.c_float else 4 for _, t in rest]
        packed = pack(*values)
        assert len(packed) == C.sizeof(whole)
        w = whole.from_buffer_copy(packed)
        assert [getattr(w.cache, n) for n, _ in cache_fields] + [getattr(w, n) for n, _ in rest] == values


def test_null_descriptors_are_refused():
    for f in (ops._L().hydra_op_cache_append, ops._L().hydra_op_cache_attention):
        assert f(None, None) == 1
    assert ops._L().hydra_op_cache_attention_ws_bytes(None, 4) == 0


def test_cache_record_checks_its_tensors():
    import torch
    k = [torch.zeros((5, 2, 16, 64), dtype=torch.int8)]
    s, t = [torch.zeros((5, 2))], torch.zeros((3, 2), dtype=torch.int32)
    ops.Cache(0, k, k, s, s, t)
    wide = torch.zeros((5, 3, 2, 16, 64), dtype=torch.int8)                            # three layers in one tensor
    c = ops.Cache(0, [wide[:, 1]], [wide[:, 1]], s, s, t)
    assert c._stride == 3 * 2 * 16 * 64
    for bad in (dict(k=[k[0].float()]), dict(k=[k[0].transpose(2, 3)]), dict(v=[k[0][:4]]), dict(k_scale=[s[0].half()]), dict(v_scale=[s[0].t()]),
                dict(page_table=t.long()), dict(page_table=t[0]), dict(k=k + k)):
        a = dict(k=k, v=k, k_scale=s, v_scale=s, page_table=t)
        a.update(bad)
        with pytest.raises(ValueError):
            ops.Cache(0, **a)


@pytest.mark.parametrize("DH", [64, 128])
def test_scratch_of_several_models_lies_in_one_allocation(DH):
    """Odd rows, heads and runs: each model's part of one buffer is on the alignment that a call asks for."""
    seen = set()
    for H in (1, 2, 3, 5):
        for n in (1, 3):
            for length in (700, 1000, 1500, 9000):
                d = cache(G=3, B=n, HKV=1, DH=DH, n_tok=n, max_pages=1000, max_len=length)[0]
                size = ops._L().hydra_op_cache_attention_ws_bytes(ops._cache_desc(*d), H)
                seen.add(size % 16)
    assert seen == {0}


def test_decoders_of_odd_sizes_cut_scratch_that_attention_takes():
    """The scratch of generate.Decoders for one head and one sequence, split into three runs."""
    from hydra_workloads import configs as C
    from oracle import model as OM
    from paper_2107_06469_amd import generate as G
    arch = C.transformer_arch(C.KIND_DECODER, 1, 128, 1, 192, 301, 768, 0, C.DTYPE_BF16)
    d = G.Decoders(arch, [OM.init_params(arch, 11, 0)] * 2, 1, 768, page=16, graph=False, device="cpu")
    ws = d._single["ws"]
    assert ws[0].numel() > 0 and (ws[1].data_ptr() - ws[0].data_ptr()) % 16 == 0


# ---- what the bindings refuse by themselves: tables and arrays that the C side knows by their addresses alone -------------------------


def two_models(**kw):
    import torch
    k = [torch.zeros((5, 2, 16, 64), dtype=torch.int8) for _ in range(2)]
    a = dict(kind=0, k=k, v=k, k_scale=[torch.zeros((5, 2))] * 2, v_scale=[torch.zeros((5, 2))] * 2, page_table=torch.zeros((3, 2), dtype=torch.int32))
    return ops.Cache(**{**a, **kw})


def test_cache_record_checks_types_and_pages():
    import torch
    for bad in (dict(page_table=torch.zeros((3, 2))), dict(k_scale=[torch.zeros((5, 2), dtype=torch.int32)] * 2),
                dict(v_scale=[torch.zeros((5, 2), dtype=torch.int32)] * 2),
                dict(k=[torch.zeros((1, 2, 16, 64), dtype=torch.int8).expand(5, 2, 16, 64)] * 2,     # all pages in one place
                     v=[torch.zeros((1, 2, 16, 64), dtype=torch.int8).expand(5, 2, 16, 64)] * 2)):
        with pytest.raises(ValueError):
            two_models(**bad)
    one = [torch.zeros((1, 2, 16, 64), dtype=torch.int8)] * 2
    two_models(k=one, v=one, k_scale=[torch.zeros((1, 2))] * 2, v_scale=[torch.zeros((1, 2))] * 2)


@pytest.mark.parametrize("bad", ["qkv", "q", "o", "lse", "ws", "lens64", "lens_float", "lens_short", "lens_strided", "ptr64", "ptr_short"])
@pytest.mark.parametrize("op", ["append", "attention"])
def test_calls_are_checked_against_their_cache(op, bad, monkeypatch):
    import torch
    monkeypatch.setattr(ops, "_stream", lambda: 0)
    c = two_models()
    x = lambda n=2, w=384, t=torch.bfloat16: [torch.zeros((3, w), dtype=t) for _ in range(n)]  # noqa: E731
    lens, ptr = torch.ones(3, dtype=torch.int32), torch.arange(4, dtype=torch.int32)
    lens = {"lens64": lens.long(), "lens_float": lens.float(), "lens_short": lens[:2], "lens_strided": torch.ones(6, dtype=torch.int32)[::2]}.get(bad, lens)
    ptr = {"ptr64": ptr.long(), "ptr_short": ptr[:3]}.get(bad, ptr)
    n = lambda name: 1 if bad == name else 2  # noqa: E731
    call = dict(q_ptr=ptr, n_tok=3, max_q=1)
    if op == "append":
        if bad in ("o", "lse", "ws"):
            return
        with pytest.raises(ValueError):
            ops.hydra_op_cache_append(c, lens, 2, 384, 128, x(n("qkv")), x(n("q"), 128), **call)
    else:
        if bad == "qkv":
            return
        with pytest.raises(ValueError):
            ops.hydra_op_cache_attention(c, lens, 2, 128, 128, True, 0.1, x(n("q"), 128), x(n("o"), 128), x(n("lse"), 2, torch.float32),
                                         ws=x(n("ws"), 64, torch.uint8), **call)


@pytest.mark.parametrize("bad", ["u", "token", "logprob", "top_k64", "temperature64", "top_p_int", "min_p_short", "token64", "top_k_strided"])
def test_draws_are_checked(bad, monkeypatch):
    import torch
    monkeypatch.setattr(ops, "_stream", lambda: 0)
    n = lambda name: 1 if bad == name else 2  # noqa: E731
    z = [torch.zeros((3, 50))] * 2
    rule = dict(t=torch.ones(3), k=torch.ones(3, dtype=torch.int32), p=torch.ones(3), m=torch.zeros(3))
    rule.update({"top_k64": dict(k=torch.ones(3, dtype=torch.int64)), "temperature64": dict(t=torch.ones(3, dtype=torch.float64)),
                 "top_p_int": dict(p=torch.ones(3, dtype=torch.int32)), "min_p_short": dict(m=torch.zeros(2)),
                 "top_k_strided": dict(k=torch.ones(6, dtype=torch.int32)[::2])}.get(bad, {}))
    token = [torch.zeros(3, dtype=torch.int64 if bad == "token64" else torch.int32)] * n("token")
    with pytest.raises(ValueError):
        ops.hydra_op_sample(ops.F32, 3, 50, 50, 50, z, z[:n("u")], *rule.values(), token, [torch.zeros(3)] * n("logprob"))


def test_which_kernel_takes_a_call():
    """The kernel for few rows or the one for prompts, its waves and the runs of keys, at sizes that tests of either count on."""
    def plan(G, HKV, DH, new, total, H):
        d, keep = cache(G=G, B=len(new), HKV=HKV, DH=DH, page=16, n_tok=sum(new), max_q=max(new), max_len=max(total), max_pages=-(-max(total) // 16))
        out = (C.c_int32 * 3)()
        assert ops._L().hydra_op_cache_attention_plan(ops._cache_desc(*d), H, out) == 0
        return tuple(out)
    assert plan(1, 2, 64, [1, 3], [400, 393], 10)[0] == 16 and plan(1, 2, 128, [1, 3], [1500, 1493], 10) == (16, 8, 6)
    assert plan(1, 2, 128, [2, 1], [3000, 1900], 10)[0] == 16                          # in one run without scratch: more than 64 pages
    assert plan(1, 12, 64, [150, 100], [330, 320], 60)[:2] == plan(1, 12, 128, [150, 100], [330, 320], 60)[:2] == (128, 4)
    assert plan(1, 12, 64, [20], [18000], 60)[:2] == (128, 4)                          # more than 512
    assert plan(3, 8, 128, [200, 0, 131], [230, 50, 131], 16) == (128, 4, 1)
    assert plan(2, 4, 128, [40, 33, 0, 7], [1500, 1411, 20, 1300], 36)[:2] == (256, 8) and plan(2, 4, 128, [40, 33], [1500, 1411], 36)[0] == 16
    out = (C.c_int32 * 3)()
    assert ops._L().hydra_op_cache_attention_plan(None, 4, out) == 1 and ops._L().hydra_op_cache_attention_plan(ops._cache_desc(*cache(DH=96)[0]), 4, out) == 1
    d, keep = cache()
    assert ops._L().hydra_op_cache_attention_plan(ops._cache_desc(*d), 4, None) == 1
