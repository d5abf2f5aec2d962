"""Token ids on their way from a draw to the embedding, which takes them as they are: the launches are recorded instead of made (no GPU)."""
import numpy as np
import pytest
import torch

from hydra_workloads import configs as C
from oracle import model as OM

V, PROMPTS = 301, [[5, 6, 7], [300]]


@pytest.fixture
def decoders(monkeypatch):
    from paper_2107_06469_amd import generate as G
    seen = []

    def embed(dtype, tokens, S, d, ld, ids, tok, pos, x):
        seen.append(ids.clone())

    def sample(dtype, rows, n, ldz, ldu, z, u, t, k, p, m, token, logprob):
        for i, (a, b) in enumerate(zip(token, logprob)):                # model 1 has nothing to draw
            a.fill_(-1 if i == 1 else V - 1), b.fill_(float("-inf") if i == 1 else -1.0)
    for name in ("hydra_op_gemm", "hydra_op_layernorm_fwd", "hydra_op_cache_append", "hydra_op_cache_attention"):
        monkeypatch.setattr(G.O, name, lambda *a, **kw: None)
    monkeypatch.setattr(G.O, "hydra_op_embed_fwd", embed)
    monkeypatch.setattr(G.O, "hydra_op_sample", sample)
    arch = C.transformer_arch(C.KIND_DECODER, 1, 128, 2, 192, V, 40, 0, C.DTYPE_BF16)
    params = [OM.init_params(arch, 11, k) for k in range(3)]
    return G.Decoders(arch, params, len(PROMPTS), 16, page=16, graph=False, device="cpu"), seen


def test_a_model_without_a_token_to_draw(decoders):
    d, seen = decoders
    tokens, logprob = d.generate(PROMPTS, 4)
    assert len(seen) == 4 * 3                                          # the prompts, then three steps, for three models
    assert all(int(ids.min()) >= 0 and int(ids.max()) < V for ids in seen)
    assert (tokens[1] == -1).all() and np.isneginf(logprob[1]).all()
    assert (tokens[[0, 2]] == V - 1).all() and all((seen[3 + 3 * s + k] == V - 1).all() for s in range(3) for k in (0, 2))


@pytest.mark.parametrize("bad", [[[-1, 3]] * 3, [[3, V]] * 3, [[2 ** 31 - 1, 0]] * 3, np.full((3, 2), -1), np.zeros((0, 2))], ids=str)
def test_steps_refuse_tokens_outside_the_vocabulary(decoders, bad):
    d, seen = decoders
    d.prefill(PROMPTS)
    n = len(seen)
    with pytest.raises(ValueError):
        d.step(bad)
    assert len(seen) == n
    d.step([[0, V - 1]] * 3)
    assert all(ids.tolist() == [0, V - 1] for ids in seen[n:]) and len(seen) == n + 3
