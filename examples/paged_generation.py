#!/usr/bin/env python3
"""Text generation with the trained layer's weights: a paged cache of keys and values, prompts read in pieces, then token by token.

    python examples/paged_generation.py

The same decoder layers that dlayer_forward and dlayer_backward train, run for tokens that come a few at a time: per layer

    h = RMSNorm(x);  q, k, v = h Wq^T, h Wk^T, h Wv^T;  kv_cache_append (rotates q and k, puts k and v into their pages)
    y1 = x + paged_attention(q) Wo^T;  y = y1 + SwiGLU MLP(RMSNorm(y1))

Rows have different lengths, and pages of 16 tokens are handed out as a row grows.  token_logprobs_forward says how likely what was chosen is, and
what else would have been.  At the end whole rows go through dlayer_forward, as in training, and the log-probabilities are compared.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2602_08387_amd as K  # noqa: E402
from synth import inputs as si  # noqa: E402

PAGE = 16


def _scratch(nbytes):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")


def _like(x, features):
    return torch.empty((x.shape[0], features), dtype=torch.bfloat16, device="cuda")


class Model:
    """Layers of cfg's widths with random weights, an embedding and an LM head."""

    def __init__(self, cfg, n_layers, vocab, seed=0):
        self.cfg, self.vocab, gen = cfg, vocab, torch.Generator().manual_seed(seed)
        normal = lambda std, *shape: (torch.randn(shape, generator=gen) * std).to(torch.bfloat16).cuda()  # noqa: E731
        ones = lambda n: torch.ones(n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.embed, self.w_lm, self.g_final = normal(1.0, vocab, cfg.d_model), normal(3.0 * cfg.d_model ** -0.5, vocab, cfg.d_model), ones(cfg.d_model)
        shapes = si.weight_shapes(cfg)
        self.layers = [{n: ones(*shapes[n]) if len(shapes[n]) == 1 else normal(shapes[n][1] ** -0.5, *shapes[n]) for n in si.WEIGHT_NAMES} for _ in range(n_layers)]

    def logits(self, x):
        """x [T, D] -> [T, vocab]."""
        T, D = x.shape
        h, rstd, out = _like(x, D), torch.empty(T, dtype=torch.float32, device="cuda"), _like(x, self.vocab)
        K.rmsnorm_forward(x, self.g_final, T, D, self.cfg.rms_eps, h, rstd)
        K.linear_forward(h, self.w_lm, None, T, D, self.vocab, out)
        return out

    def embedding(self, ids):
        """ids, any shape -> [ids, D]."""
        x = torch.empty((ids.numel(), self.cfg.d_model), dtype=torch.bfloat16, device="cuda")
        K.embed_forward(self.embed, ids.reshape(-1).contiguous(), ids.numel(), self.vocab, self.cfg.d_model, x)
        return x

    def whole_rows(self, ids):
        """ids [B, S], S a multiple of 128, through the training step's forward: [B * S, vocab]."""
        cfg, x = self.cfg.with_(batch=ids.shape[0], seq=ids.shape[1]), self.embedding(ids)
        saved, ws = _scratch(K.dlayer_saved_bytes(cfg)), _scratch(K.dlayer_workspace_bytes(cfg))
        for w in self.layers:
            y = torch.empty_like(x)
            K.dlayer_forward(cfg, x, w, y, saved, ws)
            x = y
        return self.logits(x)


class Generator:
    """Rows of tokens that grow: each layer's cache, one page table for all layers, and the pages that are still free."""

    def __init__(self, model, batch, max_tokens, e4m3=False):
        cfg, columns = model.cfg, -(-max_tokens // PAGE)
        n_pages = batch * columns
        self.model, self.table = model, torch.full((batch, columns), -1, dtype=torch.int32, device="cuda")
        self.free, self.held = list(range(n_pages))[::-1], [0] * batch
        self.tokens = torch.zeros(batch, dtype=torch.int64, device="cuda")
        shape = (n_pages, cfg.n_kv_heads, PAGE, cfg.head_dim)
        byte = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")  # noqa: E731
        if e4m3:
            self.caches = [K.KVCache.of(byte(*shape), byte(*shape), self.table, byte(*shape[:3]), byte(*shape[:3])) for _ in model.layers]
        else:
            self.caches = [K.KVCache.of(*(torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)), self.table) for _ in model.layers]

    def _pages_for(self, counts):
        for b, n in enumerate(counts):
            for column in range(-(-self.held[b] // PAGE), -(-(self.held[b] + n) // PAGE)):
                self.table[b, column] = self.free.pop()
            self.held[b] += n

    def extend(self, ids, counts):
        """The next counts[b] tokens of each row, ids [B, S] (what lies behind counts[b] is padding) -> what the layers make of them [B * S, D]."""
        cfg, (B, S) = self.model.cfg, ids.shape
        D, F, Q, KV, T = cfg.d_model, cfg.d_ff, cfg.n_q_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim, ids.numel()
        self._pages_for(counts)
        lengths = torch.tensor(counts, dtype=torch.int64, device="cuda")
        x, rstd = self.model.embedding(ids), torch.empty(T, dtype=torch.float32, device="cuda")
        ws = _scratch(K.paged_attention_workspace_bytes(self.caches[0], S, cfg.n_q_heads))
        for w, cache in zip(self.model.layers, self.caches):
            h, q, k, v, o, y1 = _like(x, D), _like(x, Q), _like(x, KV), _like(x, KV), _like(x, Q), _like(x, D)
            K.rmsnorm_forward(x, w["g_attn"], T, D, cfg.rms_eps, h, rstd)
            for name, out, n in (("wq", q, Q), ("wk", k, KV), ("wv", v, KV)):
                K.linear_forward(h, w[name], None, T, D, n, out)
            K.kv_cache_append(cache, q, k, v, self.tokens, lengths, S, cfg.n_q_heads, cfg.rope_base, cfg.rope_layout, q)
            K.paged_attention_forward(cache, q, self.tokens, lengths, S, cfg.n_q_heads, cfg.head_dim ** -0.5, o, None, ws)
            K.linear_forward(o, w["wo"], x, T, Q, D, y1)
            g, u, a, x = _like(x, F), _like(x, F), _like(x, F), _like(x, D)
            K.rmsnorm_forward(y1, w["g_mlp"], T, D, cfg.rms_eps, h, rstd)
            K.linear_swiglu_forward(h, w["w_gate"], w["w_up"], T, D, F, g, u, a)
            K.linear_forward(a, w["w_down"], y1, T, F, D, x)
        self.tokens += lengths
        return x

    def prompt(self, ids, lengths, piece=64):
        """Prompts ids [B, S] of the given lengths (at least 1), `piece` tokens of each row at a time -> logits behind each row's last token [B, vocab]."""
        last = torch.empty((len(ids), self.model.cfg.d_model), dtype=torch.bfloat16, device="cuda")
        for t in range(0, max(lengths), piece):
            counts = [min(max(n - t, 0), piece) for n in lengths]
            some = ids[:, t:t + piece].contiguous()
            x = self.extend(some, counts).view(len(ids), some.shape[1], -1)
            for b, n in enumerate(counts):
                if n and t + n == lengths[b]:
                    last[b] = x[b, n - 1]
        return self.model.logits(last)

    def generate(self, logits, n):
        """The n likeliest tokens, one after the other: (tokens, their log-probabilities, entropies, [B, n] each)."""
        B, V = logits.shape
        ws, got = _scratch(K.token_logprobs_workspace_bytes(B, V, 1)), []
        for i in range(n):
            ids, logp, entropy = (torch.empty(B, dtype=t, device="cuda") for t in (torch.int64, torch.float32, torch.float32))
            K.token_logprobs_forward(logits, None, B, V, V, 1.0, 1, None, entropy, None, ids, logp, ws)
            got.append((ids, logp, entropy))
            if i + 1 < n:
                logits = self.model.logits(self.extend(ids[:, None], [1] * B))
        return tuple(torch.stack(x, 1) for x in zip(*got))


def scores(logits, targets):
    """Log-probabilities of targets [T] under logits [T, vocab]; 0 where a target is no token."""
    T, V = logits.shape
    out = torch.empty(T, dtype=torch.float32, device="cuda")
    K.token_logprobs_forward(logits, targets, T, V, V, 1.0, 0, out, None, None, None, None, _scratch(K.token_logprobs_workspace_bytes(T, V, 0)))
    return out


def main(n_layers=4, n=48):
    cfg = si.CONFIGS["small"].with_(batch=4)
    model, gen = Model(cfg, n_layers, 4096), torch.Generator().manual_seed(1)
    lengths, whole = [37, 150, 64, 201], 256
    ids = torch.randint(model.vocab, (4, max(lengths)), generator=gen).cuda()
    for e4m3 in (False, True):
        g = Generator(model, 4, whole, e4m3)
        tokens, logp, entropy = g.generate(g.prompt(ids, lengths), n)
        rows = torch.zeros((4, whole), dtype=torch.int64, device="cuda")
        targets = torch.full((4, whole), -1, dtype=torch.int64, device="cuda")      # behind position p: the token at p + 1
        for b, m in enumerate(lengths):
            rows[b, :m], rows[b, m:m + n], targets[b, m - 1:m - 1 + n] = ids[b, :m], tokens[b], tokens[b]
        again = scores(model.whole_rows(rows), targets.view(-1)).view(4, whole)
        again = torch.stack([again[b, m - 1:m - 1 + n] for b, m in enumerate(lengths)])
        print(f"{'e4m3' if e4m3 else 'bf16'} cache: {tokens.numel()} tokens behind prompts of {lengths}, mean log-probability {float(logp.mean()):.4f}, "
              f"entropy {float(entropy.mean()):.4f}; of the whole rows at once {float(again.mean()):.4f}, differences up to {float((again - logp).abs().max()):.4f}",
              flush=True)


if __name__ == "__main__":
    main()
