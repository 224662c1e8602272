"""The small language model of examples/: its loss, gradients and logits against the fp64 oracle's operators composed the same way,
and generation from a state against the whole row at once.

Tolerances: a logit has eight roundings to bf16 behind it (h, q, k, v, their norms, o, y, f and its own), each 1.7e-3 rms, and operands that
add as much again: 6.8e-3, twice that in the 2-norm.  Gradients: the cosine bar of the layer, 0.999 for each tensor.
"""
import numpy as np
import pytest
import torch

from oracle import decoder_layer as odl
from oracle import lm_stack as olm
from oracle import token_mixing as otm
from tests.parity import COS_TOL, cosine, host_f64

pytestmark = pytest.mark.gpu

LOGITS = 1.4e-2


@pytest.fixture(scope="module")
def E():
    from examples import linear_attention_lm
    return linear_attention_lm


def _oracle(E, lm, ids, targets=None):
    """Logits [B, S, V], or (loss, gradients) with targets."""
    c, (B, S) = lm.cfg, ids.shape
    w = {n: host_f64(p) for n, p in lm.params.items()}
    wq, wk, wv = np.split(w["w_qkv"], [c.q_dim, c.q_dim + c.kv_dim])
    log_decay, T = lm.log_decay.double().cpu().numpy(), B * S
    heads = lambda t: t.reshape(B, S, -1, c.head_dim)  # noqa: E731
    flat = lambda t: t.reshape(T, -1)  # noqa: E731
    x = olm.embed_fwd(w["embed"], ids.reshape(-1))
    h, rstd = odl.rmsnorm_fwd(x, w["g_mix"], E.EPS)
    q0, k0, v = heads(h @ wq.T), heads(h @ wk.T), heads(h @ wv.T)
    q, rstd_q = otm.qk_norm_rope_fwd(q0, w["g_q"], E.EPS, E.ROPE_BASE, E.ROPE_LAYOUT)
    k, rstd_k = otm.qk_norm_rope_fwd(k0, w["g_k"], E.EPS, E.ROPE_BASE, E.ROPE_LAYOUT)
    o, _ = otm.linear_attention_fwd(q, k, v, log_decay, lm.scale)
    y = x + flat(o) @ w["w_o"].T
    f, rstd_f = odl.rmsnorm_fwd(y, w["g_final"], E.EPS)
    logits = f @ w["w_lm"].T
    if targets is None:
        return logits.reshape(B, S, -1)
    loss, dlogits, _ = olm.ce_loss_fwd_bwd(logits, targets.reshape(-1))
    g = {"w_lm": dlogits.T @ f}
    dy, g["g_final"] = odl.rmsnorm_bwd(y, w["g_final"], rstd_f, dlogits @ w["w_lm"])
    g["w_o"] = dy.T @ flat(o)
    dq, dk, dv, _ = otm.linear_attention_bwd(q, k, v, log_decay, lm.scale, heads(dy @ w["w_o"]))
    dq, g["g_q"] = otm.qk_norm_rope_bwd(q0, w["g_q"], rstd_q, dq, E.ROPE_BASE, E.ROPE_LAYOUT)
    dk, g["g_k"] = otm.qk_norm_rope_bwd(k0, w["g_k"], rstd_k, dk, E.ROPE_BASE, E.ROPE_LAYOUT)
    dqkv = np.concatenate([flat(dq), flat(dk), flat(dv)], 1)
    g["w_qkv"] = dqkv.T @ h
    dx, g["g_mix"] = odl.rmsnorm_bwd(x, w["g_mix"], rstd, dqkv @ w["w_qkv"])
    g["embed"] = olm.embed_bwd(dx + dy, ids.reshape(-1), c.vocab)
    return loss, g


def _ids(c, B, S, seed):
    return np.random.default_rng(seed).integers(0, c.vocab, (B, S))


def _norm_err(got, ref):
    return float(np.linalg.norm(got - ref) / np.linalg.norm(ref))


@pytest.mark.parametrize("B,S,Hq,Hkv,dh", [(2, 96, 4, 2, 64), (3, 64, 2, 2, 128), (1, 320, 6, 2, 32)])
def test_loss_and_gradients(E, B, S, Hq, Hkv, dh):
    lm = E.LinearAttentionLM(E.Config(256, 128, Hq, Hkv, dh), seed=S)
    tokens = _ids(lm.cfg, B, S + 1, S)
    ids, targets = (torch.from_numpy(np.ascontiguousarray(t)).cuda() for t in (tokens[:, :-1], tokens[:, 1:]))
    loss = float(lm.gradients(ids, targets))
    ref_loss, ref = _oracle(E, lm, tokens[:, :-1], tokens[:, 1:])
    assert abs(loss - ref_loss) <= 2e-3 * ref_loss, (loss, ref_loss)
    for n, g in lm.grads.items():
        assert cosine(host_f64(g), ref[n]) >= COS_TOL, n


def test_updates_lower_the_loss(E):
    lm = E.LinearAttentionLM(E.Config(256, 128, 4, 2, 64))
    tokens = torch.from_numpy(_ids(lm.cfg, 2, 65, 0)).cuda()
    losses = []
    for _ in range(10):
        losses.append(float(lm.gradients(tokens[:, :-1].contiguous(), tokens[:, 1:].contiguous())))
        lm.update(2e-3)
    assert losses[-1] < losses[0] - 0.5, losses


def test_generation_continues_prompts(E):
    """Prompts of different lengths, one of them empty of anything but its first token, then six tokens one by one."""
    lm = E.LinearAttentionLM(E.Config(256, 128, 4, 2, 64), seed=3)
    lengths, n = np.array([1, 63, 64, 100]), 6
    tokens = _ids(lm.cfg, 4, int(lengths.max()) + n, 5)
    ref = _oracle(E, lm, tokens)
    prompt = np.where(np.arange(lengths.max())[None] < lengths[:, None], tokens[:, :lengths.max()], 0)   # beyond a prompt's end: any token
    dev = torch.from_numpy(lengths).cuda()
    logits, state = lm.prompt(torch.from_numpy(prompt).cuda(), dev)
    for b, m in enumerate(lengths):
        assert _norm_err(host_f64(logits)[b, :m], ref[b, :m]) <= LOGITS, b
    rows = np.arange(4)
    for i in range(n):
        got = host_f64(lm.step(torch.from_numpy(tokens[rows, lengths + i].copy()).cuda(), state, dev + i))
        assert _norm_err(got, ref[rows, lengths + i]) <= LOGITS, i
    out = lm.generate(torch.from_numpy(prompt).cuda(), dev, n)
    assert out.shape == (4, n) and torch.equal(out[:, 0], logits[torch.arange(4), torch.from_numpy(lengths) - 1].argmax(-1))
