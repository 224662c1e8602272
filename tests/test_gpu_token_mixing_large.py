"""The norm of queries and keys and linear attention on tensors of more than 4 GiB (byte offsets past 32 bits, element offsets past 31), compared
where the offsets are largest: the last tokens of the last row, its last heads.  Decays are strong, so that a window of tokens holds what
these results depend on.  Tolerances as in test_gpu_token_mixing.
"""
import numpy as np
import pytest
import torch

from oracle import token_mixing as otm
from tests.parity import host_f64, rel_err

pytestmark = pytest.mark.gpu

ELEMENT, NORM, LINEAR_ELEMENT, STATE = 3.95e-3, 3.5e-3, 2.5e-2, 2e-6
B, S, H, DH = 2, 70001, 128, 128          # 4.6 GB in bf16
WINDOW, CHECKED, LOG_DECAY = 256, 64, -0.7   # 192 tokens before the checked ones: exp(-134)


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def _normal(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_()


def _garbage(*shape, dtype=torch.bfloat16):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def _ws(nbytes):
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device="cuda")


def _norm_err(got, ref):
    return float(np.linalg.norm(got - ref) / np.linalg.norm(ref))


def _finite(t):
    return all(bool(torch.isfinite(x).all()) for x in t.view(-1).split(1 << 28))


def _end(t, tokens):
    """The last two heads of the last row's last tokens, [1, tokens, 2, dh]."""
    return host_f64(t.view(B, S, H, DH)[-1:, -tokens:, -2:].contiguous())


def test_linear_attention(K):
    torch.manual_seed(0)
    q, k, v, do = (_normal(B * S, H, DH) for _ in range(4))
    log_decay, scale = torch.full((H,), LOG_DECAY, device="cuda"), 0.09
    o = _garbage(B * S, H, DH)
    K.linear_attention_forward(q, k, v, log_decay, None, None, B, S, H, H, DH, scale, o, None,
                               _ws(K.linear_attention_workspace_bytes(B, S, H, H, DH)))
    w = [_end(t, WINDOW) for t in (q, k, v, do)]
    decay = np.float32(LOG_DECAY).astype(np.float64) * np.ones(2)
    ref, _ = otm.linear_attention_fwd(*w[:3], decay, scale)
    assert _finite(o)
    got = _end(o, CHECKED)
    assert rel_err(got, ref[:, -CHECKED:]) <= LINEAR_ELEMENT and _norm_err(got, ref[:, -CHECKED:]) <= NORM
    del o
    grads = [_garbage(B * S, H, DH) for _ in range(3)]
    K.linear_attention_backward(q, k, v, log_decay, None, None, do, None, B, S, H, H, DH, scale, *grads, None,
                                _ws(K.linear_attention_backward_workspace_bytes(B, S, H, H, DH)))
    for name, g, r in zip(("dq", "dk", "dv"), grads, otm.linear_attention_bwd(*w[:3], decay, scale, w[3])):
        assert _finite(g), name
        got = _end(g, CHECKED)
        assert rel_err(got, r[:, -CHECKED:]) <= LINEAR_ELEMENT and _norm_err(got, r[:, -CHECKED:]) <= NORM, name


def test_qk_norm_rope(K):
    torch.manual_seed(1)
    n, eps, base = 8, 1e-5, 5e5
    x = [_normal(B * S, H, DH) for _ in range(2)]
    gains = [_normal(DH) for _ in range(2)]
    out, rstd = [_garbage(B * S, H, DH) for _ in range(2)], [_garbage(B * S, H, dtype=torch.float32) for _ in range(2)]
    K.qk_norm_rope_forward(*x, *gains, None, None, B, S, H, H, DH, eps, base, 0, *out, *rstd)
    # a gradient for the checked heads alone: those of the gains are then theirs too
    dy = [torch.zeros_like(t) for t in x]
    for t in dy:
        t.view(B, S, H, DH)[-1:, -n:, -2:] = _normal(1, n, 2, DH)
    dx, dg = [_garbage(B * S, H, DH) for _ in range(2)], [_garbage(DH) for _ in range(2)]
    K.qk_norm_rope_backward(*x, *gains, *rstd, *dy, None, None, B, S, H, H, DH, base, 0, *dx, *dg, 0,
                            _ws(K.qk_norm_rope_backward_workspace_bytes(B, S, H, H, DH)))
    for i in range(2):
        y_ref, r_ref = otm.qk_norm_rope_fwd(_end(x[i], n), host_f64(gains[i]), eps, base, 0, [S - n])
        dx_ref, dg_ref = otm.qk_norm_rope_bwd(_end(x[i], n), host_f64(gains[i]), r_ref, _end(dy[i], n), base, 0, [S - n])
        assert _finite(out[i]) and rel_err(_end(out[i], n), y_ref) <= ELEMENT, i
        assert _finite(dx[i]) and rel_err(_end(dx[i], n), dx_ref) <= ELEMENT, i
        assert rel_err(host_f64(dg[i]), dg_ref) <= ELEMENT, i


def test_states(K):
    """States of 4.6 GB: a token by the chunked form, the next by the step."""
    torch.manual_seed(2)
    rows, scale = 547, 0.09
    state = _normal(rows, H, DH, DH, dtype=torch.float32)
    log_decay = torch.full((H,), -0.1, device="cuda")
    decay = np.float32(-0.1).astype(np.float64) * np.ones(2)
    last = lambda t: host_f64(t[-1:, -2:].contiguous())  # noqa: E731
    ref = last(state)
    after = _garbage(rows, H, DH, DH, dtype=torch.float32)
    ws = _ws(K.linear_attention_workspace_bytes(rows, 1, H, H, DH))
    for call in ("forward", "step"):
        q, k, v = (_normal(rows, H, DH) for _ in range(3))
        o = _garbage(rows, H, DH)
        if call == "forward":
            K.linear_attention_forward(q, k, v, log_decay, None, state, rows, 1, H, H, DH, scale, o, after, ws)
        else:
            K.linear_attention_step(q, k, v, log_decay, None, after, rows, H, H, DH, scale, o)
        o_ref, ref = otm.linear_attention_fwd(*(last(t)[:, None] for t in (q, k, v)), decay, scale, state=ref)
        assert _finite(o) and _finite(after), call
        assert rel_err(last(o), o_ref[:, 0]) <= LINEAR_ELEMENT and _norm_err(last(o), o_ref[:, 0]) <= NORM, call
        assert _norm_err(last(after), ref) <= STATE, call
