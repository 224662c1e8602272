"""The norm of queries and keys in front of the softmax attention, forward and backward, against the fp64 oracle's operators composed the same way.

Tolerances.  q and k are rounded to bf16 in between (1.7e-3 rms each): scores, of size one here, are off by 2.4e-3, so are their weights; the weights' own rounding
and that of o add 1.7e-3 each: 3.4e-3 in the 2-norm, 1e-2 is three times that.  Gradients: the cosine bar of the layer, 0.999 for each tensor.
"""
import numpy as np
import pytest
import torch

from oracle import decoder_layer as odl
from oracle import token_mixing as otm
from synth import inputs as si
from tests.parity import COS_TOL, cosine, dev_bf16, host_f64

pytestmark = pytest.mark.gpu

EPS, BASE = 1e-5, 1e4


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,layout", [(2, 256, 4, 2, 64, 0), (1, 384, 2, 2, 128, 1), (3, 128, 6, 2, 32, 0)])
def test_normalised_attention(K, B, S, Hq, Hkv, dh, layout):
    rng, shape = np.random.default_rng(S), (B, S, Hq, Hkv, dh)
    bits = lambda std, mean, *s: si.f32_to_bf16_bits((rng.standard_normal(s) * std + mean).astype(np.float32))  # noqa: E731
    raw = {"q": bits(1.28, 0, B, S, Hq, dh), "k": bits(1.28, 0, B, S, Hkv, dh), "v": bits(1, 0, B, S, Hkv, dh), "do": bits(1, 0, B, S, Hq, dh),
           "gq": bits(0.1, 1, dh), "gk": bits(0.1, 1, dh)}
    t, r = {n: dev_bf16(b) for n, b in raw.items()}, {n: si.bf16_bits_to_f64(b) for n, b in raw.items()}
    qn, kn, o = torch.empty_like(t["q"]), torch.empty_like(t["k"]), torch.empty_like(t["q"])
    rstd = [torch.empty((B, S, h), dtype=torch.float32, device="cuda") for h in (Hq, Hkv)]
    lse = torch.empty((B, Hq, S), dtype=torch.float32, device="cuda")
    K.qk_norm_rope_forward(t["q"], t["k"], t["gq"], t["gk"], None, None, *shape, EPS, BASE, layout, qn, kn, *rstd)
    K.attention_forward(qn, kn, t["v"], *shape, o, lse)
    dqn, dkn, dv = torch.empty_like(qn), torch.empty_like(kn), torch.empty_like(t["v"])
    K.attention_backward(qn, kn, t["v"], o, t["do"], lse, *shape, dqn, dkn, dv,
                         torch.empty(K.attention_backward_workspace_bytes(*shape), dtype=torch.uint8, device="cuda"))
    dgq, dgk = torch.empty_like(t["gq"]), torch.empty_like(t["gk"])
    K.qk_norm_rope_backward(t["q"], t["k"], t["gq"], t["gk"], *rstd, dqn, dkn, None, None, *shape, BASE, layout, dqn, dkn, dgq, dgk, 0,
                            torch.empty(K.qk_norm_rope_backward_workspace_bytes(*shape), dtype=torch.uint8, device="cuda"))

    q, rq = otm.qk_norm_rope_fwd(r["q"], r["gq"], EPS, BASE, layout)
    k, rk = otm.qk_norm_rope_fwd(r["k"], r["gk"], EPS, BASE, layout)
    o_ref, _ = odl.attention_fwd(q, k, r["v"])
    assert np.linalg.norm(host_f64(o) - o_ref) <= 1e-2 * np.linalg.norm(o_ref)
    dq, dk, dv_ref = odl.attention_bwd(q, k, r["v"], r["do"])
    dq, dgq_ref = otm.qk_norm_rope_bwd(r["q"], r["gq"], rq, dq, BASE, layout)
    dk, dgk_ref = otm.qk_norm_rope_bwd(r["k"], r["gk"], rk, dk, BASE, layout)
    for name, got, ref in (("dq", dqn, dq), ("dk", dkn, dk), ("dv", dv, dv_ref), ("dgamma_q", dgq, dgq_ref), ("dgamma_k", dgk, dgk_ref)):
        assert cosine(host_f64(got), ref) >= COS_TOL, name
