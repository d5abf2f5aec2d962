"""Trained decoders answer prompts: K models of one architecture, grouped as in training, over a paged cache of 8-bit keys and values.

    python -m paper_2107_06469_amd.generate K layers batch prompt_tokens new_tokens

A step of all models is one chain of grouped launches: embedding, per block LayerNorm, the QKV product, hydra_op_cache_append,
hydra_op_cache_attention, the output product with its residual, LayerNorm and the FFN, and at the end the head's product in fp32 and
hydra_op_sample.  The step's launches are captured in a HIP graph once and replayed for every further token: what changes from step to step
(tokens, lengths, positions, uniforms) lies in device memory.  The command runs K decoders of the largest workload's shape (d=4096, 32 heads,
gated FFN 11008, vocabulary 32000) cut down to `layers` blocks and prints times and rates as JSON.

Weights come from a training context (Decoders.from_context) or as arrays in the framework's order of tensors; the working dtype is bf16.
"""
from __future__ import annotations

import json
import sys
import time
from typing import Dict, List, Sequence

import numpy as np

from . import hydra as H
from . import ops as O

LN_EPS = 1e-5
KIND_DECODER = 2


class Decoders:
    """K decoders of one architecture and the cache of one batch of sequences.

    arch: the architecture record (kind decoder, head width 64 or 128); params: per model the list of its tensors in the framework's
    order; batch: sequences; max_len: tokens that a sequence may grow to (at most the position table's rows); page: tokens of a cache page;
    kind: ops.CACHE_INT8 or ops.CACHE_E4M3; graph: capture a single-token step in a HIP graph."""

    def __init__(self, arch: Dict, params: Sequence[Sequence], batch: int, max_len: int, page: int = 64, kind: int = O.CACHE_INT8,
                 graph: bool = True, device: str = "cuda:0"):
        import torch
        if arch["kind"] != KIND_DECODER or arch["d_model"] // arch["n_heads"] not in (64, 128):
            raise ValueError("Decoders takes a decoder with heads of 64 or 128 columns")
        if not 0 < max_len <= arch["max_seq"]:
            raise ValueError(f"max_len is 1..{arch['max_seq']}, the positions that the models know")
        if batch < 1 or not params:
            raise ValueError("at least one sequence and one model")
        self.arch, self.K, self.B, self.max_len, self.graph = dict(arch), len(params), batch, max_len, graph
        self.dev = torch.device(device)
        self.gated = bool(arch["ffn_gated"])
        d, F, V = arch["d_model"], arch["d_ffn"], arch["n_out"]
        per = 14 if self.gated else 12
        shapes = [(V, d), (arch["max_seq"], d)]
        block = [(d,), (d,), (3 * d, d), (3 * d,), (d, d), (d,), (d,), (d,), (F, d), (F,)] + [(F, d), (F,)] * self.gated + [(d, F), (d,)]
        shapes += block * arch["n_layers"] + [(d,), (d,), (V, d), (V,)]

        def put(tensors):
            if len(tensors) != len(shapes):
                raise ValueError(f"{len(tensors)} tensors where this architecture has {len(shapes)}")
            out = []
            for t, s in zip(tensors, shapes):
                t = torch.as_tensor(t)
                if t.numel() != int(np.prod(s)):
                    raise ValueError(f"a tensor of {t.numel()} elements where {s} is expected")
                out.append(t.to(self.dev, torch.bfloat16 if len(s) == 2 else torch.float32).reshape(s).contiguous())
            return out
        models = [put(p) for p in params]
        group = [list(ts) for ts in zip(*models)]                      # tensor -> its copy of every model
        self.tok, self.pos = group[:2]
        self.blocks = [group[2 + per * l:2 + per * (l + 1)] for l in range(arch["n_layers"])]
        self.lnf_g, self.lnf_b, self.W_head, self.b_head = group[-4:]

        heads, dh, self.max_pages = arch["n_heads"], d // arch["n_heads"], (max_len + page - 1) // page
        n_pages = batch * self.max_pages
        table = torch.arange(n_pages, dtype=torch.int32, device=self.dev).reshape(batch, self.max_pages)
        # layer, keys/values, page: the pages of all models and layers in one tensor
        pools = torch.zeros(self.K, arch["n_layers"], 2, n_pages, heads, page, dh, dtype=torch.int8, device=self.dev)
        scales = torch.zeros(self.K, arch["n_layers"], 2, n_pages, heads, device=self.dev)
        self.cache = [O.Cache(kind, *([t[k, l, i] for k in range(self.K)] for t in (pools, scales) for i in (0, 1)), table)
                      for l in range(arch["n_layers"])]
        self.cache_bytes = pools.numel() + scales.numel() * 4
        self.lens = torch.zeros(batch, dtype=torch.int32, device=self.dev)
        self.tokens = self._rows(batch, (), torch.int32)
        self.ld_v = (V + 7) // 8 * 8
        self.logits = self._rows(batch, (self.ld_v,), torch.float32)
        self._single = self._buffers(batch, 1)
        self._step_graph, self._longest = None, 0

    @classmethod
    def from_context(cls, ctx: "H.Context", arch: Dict, models: Sequence[int], batch: int, max_len: int, **kw):
        """The models of a training context as they stand now; all of architecture `arch`."""
        return cls(arch, [H.hydra_read_params(ctx, k) for k in models], batch, max_len, **kw)

    def _rows(self, n, shape, dtype):
        import torch
        return torch.zeros(self.K, n, *shape, dtype=dtype, device=self.dev)

    def _buffers(self, n, max_q):
        """What one call of n rows writes on its way."""
        import torch
        a, bf = self.arch, torch.bfloat16
        d, F = a["d_model"], a["d_ffn"]
        b = dict(n=n, max_q=max_q)
        for name, width in (("x", d), ("y", d), ("a", d), ("qkv", 3 * d), ("h", F)) + ((("g", F),) if self.gated else ()):
            b[name] = self._rows(n, (width,), bf)
            b[name + "s"] = list(b[name])
        b["mean"], b["rstd"] = list(self._rows(n, (), torch.float32)), list(self._rows(n, (), torch.float32))
        b["last"] = self._rows(self.B, (d,), bf)
        size = O.hydra_op_cache_attention_ws_bytes(self.cache[0], a["n_heads"], n_tok=n, max_q=max_q, max_len=self.max_len)
        b["ws"] = list(self._rows(size, (), torch.uint8)) if size else None
        return b

    def _norm(self, b, n, src, dst, gamma, beta):
        d = self.arch["d_model"]
        O.hydra_op_layernorm_fwd(O.BF16, n, d, d, LN_EPS, src, dst, gamma, beta, b["mean"], b["rstd"])

    def _linear(self, n, X, W, bias, out, ldo, **kw):
        N, K = W[0].shape
        O.hydra_op_gemm(O.BF16, n, N, K, X, W, out, x_kmajor=True, w_kmajor=True, ldx=K, ldw=K, ldo=ldo, bias=bias, **kw)

    def _forward(self, b, ids, positions, q_ptr=None, last=None):
        """ids per model and positions of b["n"] rows -> self.logits of the row that ends each sequence (rows `last`; None: every row)."""
        import torch
        n, d, F, heads = b["n"], self.arch["d_model"], self.arch["d_ffn"], self.arch["n_heads"]
        dh = d // heads
        at = dict(q_ptr=q_ptr, n_tok=n, max_q=b["max_q"], max_len=self.max_len)
        for k in range(self.K):                                        # models differ in their ids from the first drawn token on
            O.hydra_op_embed_fwd(O.BF16, n, n, d, d, ids[k], [self.tok[k]], [self.pos[k].index_select(0, positions)], [b["xs"][k]])
        for cache, p in zip(self.cache, self.blocks):
            ln1g, ln1b, Wqkv, bqkv, Wo, bo, ln2g, ln2b, W1, b1 = p[:10]
            self._norm(b, n, b["xs"], b["as"], ln1g, ln1b)
            self._linear(n, b["as"], Wqkv, bqkv, b["qkvs"], 3 * d)
            O.hydra_op_cache_append(cache, self.lens, heads, 3 * d, 0, b["qkvs"], **at)
            # the queries are read where the product left them, in the first columns of qkv's rows
            O.hydra_op_cache_attention(cache, self.lens, heads, 3 * d, d, True, dh ** -0.5, b["qkvs"], b["as"], ws=b["ws"], **at)
            self._linear(n, b["as"], Wo, bo, b["ys"], d, resid=b["xs"], ldr=d)
            self._norm(b, n, b["ys"], b["as"], ln2g, ln2b)
            if self.gated:
                self._linear(n, b["as"], p[10], p[11], b["gs"], F, act=O.EPI_GELU)
                self._linear(n, b["as"], W1, b1, b["hs"], F)
                torch.mul(b["h"], b["g"], out=b["h"])
            else:
                self._linear(n, b["as"], W1, b1, b["hs"], F, act=O.EPI_GELU)
            self._linear(n, b["hs"], p[-2], p[-1], b["xs"], d, resid=b["ys"], ldr=d)
        x = b["x"]
        if last is not None:
            torch.index_select(x, 1, last, out=b["last"])
            x = b["last"]
        self._norm(b, self.B, list(x), b["as"], self.lnf_g, self.lnf_b)
        self._linear(self.B, b["as"], self.W_head, self.b_head, list(self.logits), self.ld_v, out_f32=True)

    def prefill(self, prompts: Sequence[Sequence[int]]):
        """Starts the batch's sequences anew from one non-empty prompt each (lengths may differ), the same for every model; returns the logits
        [K, batch, V] of the token after each."""
        import torch
        if len(prompts) != self.B or min(len(p) for p in prompts) < 1 or max(len(p) for p in prompts) > self.max_len:
            raise ValueError(f"{self.B} prompts of 1..{self.max_len} tokens each")
        n = [len(p) for p in prompts]
        flat = np.concatenate([np.asarray(p, dtype=np.int32) for p in prompts])
        if flat.min() < 0 or flat.max() >= self.arch["n_out"]:
            raise ValueError(f"a token outside 0..{self.arch['n_out'] - 1}")
        ends = np.cumsum(n)
        up = lambda x, t: torch.as_tensor(np.asarray(x)).to(self.dev, t)
        self.lens.copy_(up(n, torch.int32))
        self._forward(self._buffers(len(flat), max(n)), [up(flat, torch.int32)] * self.K, up(np.concatenate([np.arange(m) for m in n]), torch.int64),
                      up(np.concatenate([[0], ends]), torch.int32), up(ends - 1, torch.int64))
        self._longest = max(n)
        return self.logits[..., :self.arch["n_out"]]

    def _single_step(self):
        import torch
        positions = self.lens.to(torch.int64)
        self.lens.add_(1)
        # a model without a token to draw (its logits are no numbers) has -1 here and goes on from token 0: the embedding takes ids as they are
        self._forward(self._single, list(self.tokens.clamp(0, self.arch["n_out"] - 1)), positions)

    def step(self, tokens=None):
        """One token more per sequence: tokens [K, batch] of the vocabulary (looked at on the host; None: the ones in self.tokens, as they were drawn);
        returns the next logits [K, batch, V]."""
        import torch
        if self._longest >= self.max_len:
            raise ValueError(f"a sequence has all of its {self.max_len} tokens")
        if tokens is not None:
            tokens = torch.as_tensor(tokens)
            if not (tokens.numel() and 0 <= int(tokens.min()) and int(tokens.max()) < self.arch["n_out"]):
                raise ValueError(f"a token outside 0..{self.arch['n_out'] - 1}")
            self.tokens.copy_(tokens)
        self._longest += 1
        if not self.graph:
            self._single_step()
        elif self._step_graph is None:
            self._single_step()                                        # the first one as it is: the library sets itself up on first use
            torch.cuda.synchronize(self.dev)
            self._step_graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self._step_graph):                   # recorded, not run
                self._single_step()
        else:
            self._step_graph.replay()
        return self.logits[..., :self.arch["n_out"]]

    def generate(self, prompts: Sequence[Sequence[int]], new_tokens: int, temperature: float = 1.0, top_k: int = 0, top_p: float = 1.0,
                 min_p: float = 0.0, seed: int = 0):
        """new_tokens drawn tokens per model and sequence and the log-probabilities that the model gave them: two arrays
        [K, batch, new_tokens].  temperature 0 takes the largest logit.  A model whose logits are no numbers has nothing to draw: -1 and -inf from there
        on, the other models' tokens are what they would be without it."""
        import torch
        V, B = self.arch["n_out"], self.B
        if new_tokens < 1 or max(len(p) for p in prompts) + new_tokens - 1 > self.max_len:
            raise ValueError(f"prompts and new tokens have room for {self.max_len} tokens")
        rule = [torch.full((B,), x, dtype=t, device=self.dev) for x, t in
                ((temperature, torch.float32), (top_k, torch.int32), (top_p, torch.float32), (min_p, torch.float32))]
        gen = torch.Generator(self.dev).manual_seed(seed)
        u, logprob = self._rows(B, (V,), torch.float32), self._rows(B, (), torch.float32)
        drawn, given = self._rows(B, (new_tokens,), torch.int32), self._rows(B, (new_tokens,), torch.float32)
        self.prefill(prompts)
        for i in range(new_tokens):
            if i:
                self.step()
            u.uniform_(generator=gen)
            O.hydra_op_sample(O.F32, B, V, self.ld_v, V, list(self.logits), list(u), *rule, list(self.tokens), list(logprob))
            drawn[..., i], given[..., i] = self.tokens, logprob
        return drawn.cpu().numpy(), given.cpu().numpy()


def run(K: int, layers: int, batch: int, prompt: int, new: int) -> Dict:
    """K decoders of the largest workload's shape with `layers` blocks, random weights: times of the prompts and of a step."""
    import torch
    from hydra_workloads import workload
    w = workload(4)
    arch = dict(w.archs[0], n_layers=layers)
    ctx = H.hydra_create(n_streams=1)
    try:
        H.hydra_define_models(ctx, [arch] * K, w.hparams[:K], w.init_seed)
        for k in range(K):
            H.hydra_shard(ctx, k, [])
        d = Decoders.from_context(ctx, arch, range(K), batch, prompt + new)
    finally:
        H.hydra_destroy(ctx)
        torch.cuda.empty_cache()
    prompts = np.random.default_rng(w.data_seed).integers(0, arch["n_out"], size=(batch, prompt))
    first = d.generate(prompts, min(new, 3), top_k=50, seed=1)        # the step's graph is captured here
    torch.cuda.synchronize()
    t0 = time.time()
    d.prefill(prompts)
    torch.cuda.synchronize()
    t1 = time.time()
    tokens, logprob = d.generate(prompts, new, top_k=50, seed=1)
    t2 = time.time()
    step = (t2 - t1 - (t1 - t0)) / max(new - 1, 1)
    weights = sum(t.numel() * t.element_size() for p in d.blocks for g in p for t in g) + sum(t.numel() * 2 for t in d.W_head)
    return dict(models=K, layers=layers, batch=batch, prompt=prompt, new=new, prefill_ms=(t1 - t0) * 1e3, step_ms=step * 1e3,
                tokens_per_s=K * batch / step, weights_GB=weights / 1e9, cache_GB=d.cache_bytes / 1e9,
                weight_read_TBps=weights / step / 1e12, repeatable=bool(np.array_equal(first[0], tokens[..., :first[0].shape[-1]])),
                mean_logprob=float(logprob.mean()))


def main(argv):
    n = [int(x) for x in argv[1:]] + [2, 4, 8, 1024, 64][len(argv) - 1:]
    print(json.dumps(run(*n)), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main(sys.argv))
