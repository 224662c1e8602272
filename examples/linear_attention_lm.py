#!/usr/bin/env python3
"""A small language model that mixes tokens by linear attention: trained, then prompted and run token by token.

    python examples/linear_attention_lm.py

One block between an embedding and an LM head, all of it the library's kernels (torch holds the memory, puts the gradients of q, k and v side by side and picks the likeliest token):

    h = RMSNorm(x);  q, k, v = h Wq^T, h Wk^T, h Wv^T;  q, k <- qk_norm_rope(q, k);  y = x + linear_attention(q, k, v) Wo^T

Training runs qk_norm_rope and linear_attention forward and backward over rows of one length.  Generation reads prompts of different
lengths in one call, which leaves the state behind each row's last token, and goes on from there with linear_attention_step: a
token costs the same however many came before it, and the state [Hkv, dh, dh] takes the place of a cache that grows.
"""
from __future__ import annotations

import dataclasses
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2602_08387_amd as K  # noqa: E402

EPS, ROPE_BASE, ROPE_LAYOUT = 1e-5, 1e4, 0


@dataclasses.dataclass(frozen=True)
class Config:
    vocab: int = 512
    d_model: int = 256
    n_q_heads: int = 8
    n_kv_heads: int = 4
    head_dim: int = 64

    @property
    def q_dim(self):
        return self.n_q_heads * self.head_dim

    @property
    def kv_dim(self):
        return self.n_kv_heads * self.head_dim


def _scratch(nbytes):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")


class LinearAttentionLM:
    def __init__(self, cfg: Config, seed=0):
        self.cfg, gen = cfg, torch.Generator().manual_seed(seed)
        normal = lambda std, *shape: (torch.randn(shape, generator=gen) * std).to(torch.bfloat16).cuda()  # noqa: E731
        ones = lambda n: torch.ones(n, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        D = cfg.d_model
        self.params = {
            "embed": normal(1.0, cfg.vocab, D),
            "g_mix": ones(D),
            "w_qkv": normal(D ** -0.5, cfg.q_dim + 2 * cfg.kv_dim, D),   # rows of Wq, Wk, Wv: each is a matrix of its own, the three are one
            "g_q": ones(cfg.head_dim),
            "g_k": ones(cfg.head_dim),
            "w_o": normal(cfg.q_dim ** -0.5, D, cfg.q_dim),
            "g_final": ones(D),
            "w_lm": normal(D ** -0.5, cfg.vocab, D),
        }
        self.grads = {n: torch.empty_like(p) for n, p in self.params.items()}
        self.moments = [[torch.zeros(p.shape, dtype=torch.float32, device="cuda") for p in self.params.values()] for _ in range(2)]
        # half-lives of 11 tokens for the first head up to 11 * 2^(n-1) for the last
        self.log_decay = torch.tensor([math.log1p(-2.0 ** -(4 + j)) for j in range(cfg.n_kv_heads)], dtype=torch.float32, device="cuda")
        self.scale = 1.0 / cfg.head_dim
        self.steps = 0

    def _buffer(self, *shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def _project(self, ids, T):
        """Embedding, norm and the three projections of T tokens, and what the backward needs of them."""
        c, p = self.cfg, self.params
        x, h, rstd = self._buffer(T, c.d_model), self._buffer(T, c.d_model), self._buffer(T, dtype=torch.float32)
        K.embed_forward(p["embed"], ids, T, c.vocab, c.d_model, x)
        K.rmsnorm_forward(x, p["g_mix"], T, c.d_model, EPS, h, rstd)
        out = []
        for w in p["w_qkv"].split([c.q_dim, c.kv_dim, c.kv_dim]):
            out.append(self._buffer(T, w.shape[0]))
            K.linear_forward(h, w, None, T, c.d_model, w.shape[0], out[-1])
        return x, h, rstd, out

    def _finish(self, x, o, T):
        """Output projection with the residual, and the final norm."""
        c, p = self.cfg, self.params
        y, f, rstd = self._buffer(T, c.d_model), self._buffer(T, c.d_model), self._buffer(T, dtype=torch.float32)
        K.linear_forward(o, p["w_o"], x, T, c.q_dim, c.d_model, y)
        K.rmsnorm_forward(y, p["g_final"], T, c.d_model, EPS, f, rstd)
        return y, f, rstd

    def _shape(self, B, S):
        return B, S, self.cfg.n_q_heads, self.cfg.n_kv_heads, self.cfg.head_dim

    def gradients(self, ids, targets):
        """ids, targets [B, S] int64 -> the mean loss, a tensor of one; the gradients of all parameters are left in self.grads.  B S is a multiple
        of 64."""
        (B, S), c, p, g = ids.shape, self.cfg, self.params, self.grads
        T, shape, D = B * S, self._shape(B, S), c.d_model
        x, h, rstd, (q0, k0, v) = self._project(ids, T)
        q, k, o = torch.empty_like(q0), torch.empty_like(k0), torch.empty_like(q0)
        rstd_q, rstd_k = self._buffer(T, c.n_q_heads, dtype=torch.float32), self._buffer(T, c.n_kv_heads, dtype=torch.float32)
        K.qk_norm_rope_forward(q0, k0, p["g_q"], p["g_k"], None, None, *shape, EPS, ROPE_BASE, ROPE_LAYOUT, q, k, rstd_q, rstd_k)
        K.linear_attention_forward(q, k, v, self.log_decay, None, None, *shape, self.scale, o, None,
                                   _scratch(K.linear_attention_workspace_bytes(*shape)))
        y, f, rstd_f = self._finish(x, o, T)

        loss, df = self._buffer(1, dtype=torch.float32), torch.empty_like(f)
        K.lm_head_ce_fwd_bwd(f, p["w_lm"], targets, T, D, c.vocab, 1.0, 0, loss, df, g["w_lm"], 0,
                             _scratch(K.lm_head_ce_workspace_bytes(T, D, c.vocab)))
        dy, do, dh, dx = torch.empty_like(y), torch.empty_like(o), torch.empty_like(h), torch.empty_like(x)
        norm_ws = _scratch(K.rmsnorm_backward_workspace_bytes(T, D))
        K.rmsnorm_backward(y, p["g_final"], rstd_f, df, None, T, D, dy, g["g_final"], 0, norm_ws)
        K.linear_backward(o, p["w_o"], dy, T, c.q_dim, D, do, g["w_o"], 0, _scratch(K.linear_backward_workspace_bytes(T, c.q_dim, D)))
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        K.linear_attention_backward(q, k, v, self.log_decay, None, None, do, None, *shape, self.scale, dq, dk, dv, None,
                                    _scratch(K.linear_attention_backward_workspace_bytes(*shape)))
        K.qk_norm_rope_backward(q0, k0, p["g_q"], p["g_k"], rstd_q, rstd_k, dq, dk, None, None, *shape, ROPE_BASE, ROPE_LAYOUT, dq, dk,
                                g["g_q"], g["g_k"], 0, _scratch(K.qk_norm_rope_backward_workspace_bytes(*shape)))
        n_qkv = c.q_dim + 2 * c.kv_dim
        K.linear_backward(h, p["w_qkv"], torch.cat([dq, dk, dv], 1), T, D, n_qkv, dh, g["w_qkv"], 0,
                          _scratch(K.linear_backward_workspace_bytes(T, D, n_qkv)))
        K.rmsnorm_backward(x, p["g_mix"], rstd, dh, dy, T, D, dx, g["g_mix"], 0, norm_ws)
        K.embed_backward(dx, ids, T, c.vocab, D, g["embed"], _scratch(K.embed_backward_workspace_bytes(T, c.vocab)))
        return loss

    def update(self, lr):
        params, grads = list(self.params.values()), list(self.grads.values())
        sq_norm = self._buffer(1, dtype=torch.float32)
        K.grad_sq_norm(grads, sq_norm, 0, _scratch(K.grad_sq_norm_workspace_bytes(grads)))
        self.steps += 1
        K.adamw_step(params, grads, *self.moments, self.steps, lr, 0.9, 0.95, 1e-8, 0.0, 1.0, sq_norm)

    def _logits(self, f, T):
        logits = self._buffer(T, self.cfg.vocab)
        K.linear_forward(f, self.params["w_lm"], None, T, self.cfg.d_model, self.cfg.vocab, logits)
        return logits

    def prompt(self, ids, lengths=None):
        """ids [B, S], lengths [B] -> logits [B, S, vocab] and the state behind each row's last token."""
        (B, S), c, p = ids.shape, self.cfg, self.params
        T, shape = B * S, self._shape(B, S)
        x, _, _, (q, k, v) = self._project(ids, T)
        o, state = torch.empty_like(q), self._buffer(B, c.n_kv_heads, c.head_dim, c.head_dim, dtype=torch.float32)
        K.qk_norm_rope_forward(q, k, p["g_q"], p["g_k"], None, lengths, *shape, EPS, ROPE_BASE, ROPE_LAYOUT, q, k, None, None)
        K.linear_attention_forward(q, k, v, self.log_decay, lengths, None, *shape, self.scale, o, state,
                                   _scratch(K.linear_attention_workspace_bytes(*shape)))
        return self._logits(self._finish(x, o, T)[1], T).view(B, S, c.vocab), state

    def step(self, ids, state, positions):
        """One more token for each row: ids [B], at positions [B]; the state is updated -> logits [B, vocab]."""
        (B,), c, p = ids.shape, self.cfg, self.params
        x, _, _, (q, k, v) = self._project(ids, B)
        o = torch.empty_like(q)
        K.qk_norm_rope_forward(q, k, p["g_q"], p["g_k"], positions, None, *self._shape(B, 1), EPS, ROPE_BASE, ROPE_LAYOUT, q, k, None, None)
        K.linear_attention_step(q, k, v, self.log_decay, None, state, B, c.n_q_heads, c.n_kv_heads, c.head_dim, self.scale, o)
        return self._logits(self._finish(x, o, B)[1], B)

    def generate(self, ids, lengths, n):
        """The n likeliest tokens, one after the other, behind prompts ids [B, S] of the given lengths (at least 1): [B, n]."""
        logits, state = self.prompt(ids, lengths)
        last = logits[torch.arange(len(ids), device="cuda"), lengths - 1]
        out = [last.argmax(-1)]
        for i in range(n - 1):
            out.append(self.step(out[-1], state, lengths + i).argmax(-1))
        return torch.stack(out, 1)


def periodic_rows(cfg, B, S, period, gen):
    """B rows of S tokens, each `period` random ones over and over."""
    return torch.randint(cfg.vocab, (B, period), generator=gen).repeat(1, -(-S // period))[:, :S].cuda()


def main(steps=600, period=16):
    cfg, gen = Config(), torch.Generator().manual_seed(1)
    lm = LinearAttentionLM(cfg)
    for i in range(steps):
        rows = periodic_rows(cfg, 64, 129, period, gen)
        loss = lm.gradients(rows[:, :-1].contiguous(), rows[:, 1:].contiguous())
        lm.update(2e-3)
        if i % 100 == 0 or i == steps - 1:
            # (the first tokens of a row cannot be known)
            print(f"step {i:4d}  loss {float(loss):.4f}  (at first {math.log(cfg.vocab):.2f}, at best {(period - 1) / 128 * math.log(cfg.vocab):.2f})",
                  flush=True)
    n, rows = 32, periodic_rows(cfg, 8, 160, period, gen)
    lengths = torch.randint(64, 129, (8,), generator=gen).cuda()
    out = lm.generate(rows[:, :128].contiguous(), lengths, n)
    want = torch.stack([rows[b, m:m + n] for b, m in enumerate(lengths.tolist())])
    print(f"generated behind prompts of {lengths.tolist()} tokens: {float((out == want).double().mean()) * 100:.1f} % of {out.numel()} tokens "
          f"go on as the row does")


if __name__ == "__main__":
    main()
