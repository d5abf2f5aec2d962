"""Trained decoders answering prompts (GPU only): K models in a group, prompts of different lengths in one call, then token by token, against
the oracle's full forward pass in 64 bits over all tokens so far.

Tolerance: relative L2 error of a row of logits.  A block rounds about six matrices to bf16 (2^-9/sqrt(3) = 0.11 % each, 0.28 % together) and reads
keys and values of 7 bits (a step of 2*3.5 sigma/254, so 0.8 % of a value, less after averaging over tokens); e4m3 has 3 bits of fraction (2^-4/
sqrt(3) = 3.6 % of a value).  Two blocks, and a factor of 2 for what softmax, gelu and LayerNorm amplify: 2*sqrt(2)*0.85 % = 2.4 % for int8, 10.3 % for
e4m3; 4 % and 12 % are allowed.  Losing one token's key or value of the 20 or so, or its position, moves a row by more (checked on the oracle)."""
import numpy as np
import pytest

from hydra_workloads import configs as C
from oracle import layers as L
from oracle import model as OM

pytestmark = pytest.mark.gpu

TOL = {0: 4e-2, 1: 12e-2}


@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    from paper_2107_06469_amd import generate
    return generate


def _models(gated, heads, K, d=128):
    """K decoders whose weights are as large as after training: scores, values and logits of the order of one."""
    arch = C.transformer_arch(C.KIND_DECODER, 2, d, heads, 192, 301, 80, gated, C.DTYPE_BF16)
    rng = np.random.default_rng(7)
    models = []
    for k in range(K):
        p = OM.init_params(arch, 11, k)
        models.append([t * 4 if t.ndim == 2 else t + 0.1 * rng.standard_normal(t.shape).astype(np.float32) for t in p])
    return arch, models


def _oracle_logits(arch, params, tokens):
    """Logits after the last of `tokens`."""
    batch = dict(inputs=np.array([tokens], dtype=np.int32), target_pos=np.array([[len(tokens) - 1]]), targets=np.zeros((1, 1), dtype=np.int32))
    x = None
    for u in range(OM.n_units(arch)):
        x, c = OM.unit_fwd(arch, params, u, x, batch)
    return L.linear_fwd(c["xt"], params[-2].astype(np.float64), params[-1].astype(np.float64))[0]


def _rel(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


PROMPT_LENGTHS = [17, 1, 33, 20]


def _prompts(n_out=301):
    rng = np.random.default_rng(3)
    return [rng.integers(0, n_out, size=n) for n in PROMPT_LENGTHS]


@pytest.mark.parametrize("gated,heads,K,kind,graph", [(1, 2, 3, 0, True), (0, 1, 1, 0, False), (1, 1, 2, 1, True)])
def test_prompts_and_steps_match_a_full_forward_pass(G, gated, heads, K, kind, graph):
    arch, models = _models(gated, heads, K)
    d = G.Decoders(arch, models, len(PROMPT_LENGTHS), 48, page=16, kind=kind, graph=graph)
    for repeat in range(2):                                            # the second time over the first one's pages and with its graph
        seqs = [[list(p) for p in _prompts()] for _ in range(K)]
        z = d.prefill(_prompts()).cpu().numpy()
        for step in range(6):
            for k in range(K):
                for b, s in enumerate(seqs[k]):
                    e = _rel(z[k, b], _oracle_logits(arch, models[k], s))
                    assert e < TOL[kind], f"model {k}, sequence {b} of {len(s)} tokens, step {step}, repeat {repeat}: {e:.4f}"
            tok = z.argmax(-1).astype(np.int32)
            for k in range(K):
                for b in range(len(seqs[k])):
                    seqs[k][b].append(int(tok[k, b]))
            z = d.step(tok).cpu().numpy()


def test_the_tolerance_notices_a_lost_token():
    arch, models = _models(1, 2, 1)
    for p in _prompts():
        if len(p) > 1:
            whole = _oracle_logits(arch, models[0], p)
            assert _rel(_oracle_logits(arch, models[0], np.r_[(p[0] + 1) % 301, p[1:]]), whole) > 2 * TOL[0]


def test_generated_tokens(G):
    arch, models = _models(1, 2, 2)
    make = lambda graph: G.Decoders(arch, models, len(PROMPT_LENGTHS), 48, page=16, graph=graph)
    d = make(True)
    tokens, logprob = d.generate(_prompts(), 9, temperature=0.0)
    for k in range(2):
        for b, p in enumerate(_prompts()):
            s = list(p)
            for t, lp in zip(tokens[k, b], logprob[k, b]):
                z = _oracle_logits(arch, models[k], s)
                # the largest of the device's logits is within twice their largest error of the oracle's largest
                assert z[t] >= z.max() - 2 * TOL[0] * np.linalg.norm(z)
                assert abs(lp - (z[t] - z.max() - np.log(np.exp(z - z.max()).sum()))) < 2 * TOL[0] * np.linalg.norm(z)
                s.append(int(t))
    again, _ = d.generate(_prompts(), 9, temperature=0.0)
    eager, _ = make(False).generate(_prompts(), 9, temperature=0.0)
    assert np.array_equal(tokens, again) and np.array_equal(tokens, eager)
    drawn = [d.generate(_prompts(), 9, temperature=1.5, top_k=40, top_p=0.95, min_p=0.01, seed=s)[0] for s in (1, 1, 2)]
    assert np.array_equal(drawn[0], drawn[1]) and not np.array_equal(drawn[0], drawn[2])
    eager = make(False).generate(_prompts(), 9, temperature=1.5, top_k=40, top_p=0.95, min_p=0.01, seed=1)[0]
    assert np.array_equal(drawn[0], eager) and drawn[0].min() >= 0 and drawn[0].max() < 301


def test_models_of_a_training_context(G):
    from paper_2107_06469_amd import hydra as H
    arch, _ = _models(1, 2, 1)
    ctx = H.hydra_create(n_streams=1)
    try:
        H.hydra_define_models(ctx, [arch] * 2, [C.hparams(C.OPT_ADAM, 1e-3)] * 2, 42)
        for k in range(2):
            H.hydra_shard(ctx, k, [])
        d = G.Decoders.from_context(ctx, arch, [1], 2, 40)
        z = d.prefill([[5, 6, 7], [8]]).cpu().numpy()
        params = H.hydra_read_params(ctx, 1)
    finally:
        H.hydra_destroy(ctx)
    for b, s in enumerate(([5, 6, 7], [8])):
        assert _rel(z[0, b], _oracle_logits(arch, [t.reshape(sh) for t, (_, sh, _) in zip(params, OM.tensor_specs(arch))], s)) < TOL[0]


def test_refusals(G):
    arch, models = _models(1, 2, 1)
    for bad in (dict(arch, kind=C.KIND_ENCODER), dict(arch, n_heads=8)):
        with pytest.raises(ValueError):
            G.Decoders(bad, models, 1, 16)
    for batch, max_len, params in ((1, 81, models), (1, 0, models), (0, 16, models), (1, 16, []), (1, 16, [models[0][:-1]])):
        with pytest.raises(ValueError):
            G.Decoders(arch, params, batch, max_len)
    d = G.Decoders(arch, models, 1, 16, page=16)
    for prompts in ([], [[]], [[1], [2]], [list(range(17))], [[301]], [[-1]]):
        with pytest.raises(ValueError):
            d.prefill(prompts)
    with pytest.raises(ValueError):
        d.generate([[1, 2]], 16)
    d.prefill([list(range(16))])
    with pytest.raises(ValueError):
        d.step()


@pytest.mark.parametrize("graph", [True, False])
def test_a_model_whose_logits_are_no_numbers(G, graph):
    """One diverged candidate of three: -1 and -inf for it, and the others' tokens as with a sound model in its place."""
    arch, models = _models(1, 2, 3)
    lost = [models[0], models[1][:-1] + [np.full_like(models[1][-1], np.nan)], models[2]]
    (want, want_lp), (got, got_lp) = (G.Decoders(arch, m, len(PROMPT_LENGTHS), 48, page=16, graph=graph).generate(_prompts(), 7, top_k=20, seed=4)
                                      for m in (models, lost))
    assert (got[1] == -1).all() and np.isneginf(got_lp[1]).all()
    assert np.array_equal(got[[0, 2]], want[[0, 2]]) and np.array_equal(got_lp[[0, 2]], want_lp[[0, 2]])
    assert want.min() >= 0
