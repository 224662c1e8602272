"""The gradient of the norm of queries and keys with the rotary embedding against differences of its own forward.

Tolerances.  The outputs are linear in the gains: both sides are sums of products whose rounding errors (1.7e-3 rms of each) are independent, six
deviations.  In the inputs, for a step of h = 0.1 of their size: the mean of the gradients at both ends leaves h^2 / 12 times third
derivatives of x / |x| (at most 6) of the difference, 5e-3; the outputs' rounding, 2.4e-3 of them, enters the difference squared where it is its own
direction, (2.4e-3 / h)^2 = 6e-4, and as noise of 2.4e-2 / sqrt(N).  1e-2.
"""
import numpy as np
import pytest
import torch

from synth import inputs as si
from tests.parity import dev_bf16, host_f64

pytestmark = pytest.mark.gpu

EPS, BASE, RMS = 1e-5, 1e4, 1.7e-3


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def _bf16(a):
    return dev_bf16(si.f32_to_bf16_bits(np.asarray(a, np.float32)))


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,layout,start", [(2, 200, 6, 2, 64, 0, [0, 31]), (1, 333, 4, 4, 128, 1, None), (3, 50, 5, 1, 32, 1, [7, 0, 9000])])
def test_gradient_against_differences(K, B, S, Hq, Hkv, dh, layout, start):
    rng = np.random.default_rng(S)
    start = None if start is None else torch.tensor(start, dtype=torch.int64, device="cuda")
    gains = [_bf16(rng.standard_normal(dh) * 0.1 + 1) for _ in range(2)]
    heads, shape = (Hq, Hkv), (B, S, Hq, Hkv, dh)
    ends = [[_bf16(rng.standard_normal((B, S, h, dh))) for h in heads]]
    ends.append([_bf16(host_f64(x) + 0.1 * rng.standard_normal(x.shape)) for x in ends[0]])

    def forward(x, g):
        y, rstd = [torch.empty_like(t) for t in x], [torch.empty(t.shape[:3], dtype=torch.float32, device="cuda") for t in x]
        K.qk_norm_rope_forward(*x, *g, start, None, *shape, EPS, BASE, layout, *y, *rstd)
        return y, rstd

    def backward(x, rstd, dy):
        dx, dg = [torch.empty_like(t) for t in x], [torch.empty_like(g) for g in gains]
        ws = torch.empty(K.qk_norm_rope_backward_workspace_bytes(*shape), dtype=torch.uint8, device="cuda")
        K.qk_norm_rope_backward(*x, *gains, *rstd, *dy, start, None, *shape, BASE, layout, *dx, *dg, 0, ws)
        return dx, dg

    out = [forward(x, gains) for x in ends]
    change = [host_f64(b) - host_f64(a) for a, b in zip(out[0][0], out[1][0])]
    dy = [_bf16(c * 10) for c in change]   # along the change: all terms of one sign
    grads = [backward(x, rstd, dy) for x, (_, rstd) in zip(ends, out)]
    for i in range(2):
        left = np.sum(change[i] * host_f64(dy[i]))
        step = host_f64(ends[1][i]) - host_f64(ends[0][i])
        right = np.sum(0.5 * (host_f64(grads[0][0][i]) + host_f64(grads[1][0][i])) * step)
        assert abs(left - right) <= 1e-2 * left, (i, left, right)
    # linear in the gains: the outputs with others in their place
    other = [_bf16(rng.standard_normal(dh)) for _ in range(2)]
    y, _ = forward(ends[0], other)
    for i in range(2):
        a, b = host_f64(y[i]) * host_f64(dy[i]), host_f64(grads[0][1][i]) * host_f64(other[i])
        assert abs(a.sum() - b.sum()) <= 6 * RMS * (np.linalg.norm(a) + np.linalg.norm(b)), i
