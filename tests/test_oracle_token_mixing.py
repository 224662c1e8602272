"""Pins of the oracle of the query and key norm and of linear attention: closed forms, the sum over pairs, finite differences."""
import numpy as np
import pytest

from oracle import token_mixing as otm


def test_norm_and_rotation_closed_forms():
    rng = np.random.default_rng(0)
    x, gamma = rng.standard_normal((2, 5, 3, 32)), 1 + 0.1 * rng.standard_normal(32)
    y, rstd = otm.qk_norm_rope_fwd(x, gamma, 1e-5, 1e4, 0)
    assert np.allclose(rstd, (np.mean(x ** 2, -1) + 1e-5) ** -0.5, rtol=1e-14)
    assert np.allclose(y[:, 0], x[:, 0] * rstd[:, 0, :, None] * gamma, rtol=1e-14)            # position 0 turns nothing
    for layout in (0, 1):
        y, _ = otm.qk_norm_rope_fwd(x, np.ones(32), 0.0, 1e4, layout)
        assert np.allclose(np.sum(y ** 2, -1), 32, rtol=1e-12)                                  # a rotation keeps the length
        later, _ = otm.qk_norm_rope_fwd(x[:, 2:], np.ones(32), 0.0, 1e4, layout, start=[2, 2])
        assert np.allclose(later, y[:, 2:], rtol=0, atol=1e-13)                                 # start is the position of the first token
    short, rstd = otm.qk_norm_rope_fwd(x, gamma, 1e-5, 1e4, 0, lengths=[0, 3])
    assert not short[0].any() and not rstd[0].any() and not short[1, 3:].any() and short[1, 2].all()


@pytest.mark.parametrize("layout", [0, 1])
def test_norm_gradient_against_differences(layout):
    rng = np.random.default_rng(layout)
    x, gamma, dy = rng.standard_normal((2, 4, 3, 32)), 1 + 0.1 * rng.standard_normal(32), rng.standard_normal((2, 4, 3, 32))
    start, lengths = [3, 70], [4, 2]
    f = lambda x, g: float(np.sum(dy * otm.qk_norm_rope_fwd(x, g, 1e-5, 1e4, layout, start, lengths)[0]))  # noqa: E731
    _, rstd = otm.qk_norm_rope_fwd(x, gamma, 1e-5, 1e4, layout, start, lengths)
    dx, dgamma = otm.qk_norm_rope_bwd(x, gamma, rstd, dy, 1e4, layout, start, lengths)
    u, w, h = rng.standard_normal(x.shape), rng.standard_normal(32), 1e-5
    assert np.isclose((f(x + h * u, gamma) - f(x - h * u, gamma)) / (2 * h), np.sum(dx * u), rtol=1e-7)
    assert np.isclose((f(x, gamma + h * w) - f(x, gamma - h * w)) / (2 * h), np.sum(dgamma * w), rtol=1e-7)
    assert not dx[1, 2:].any()


def _linear_case(seed):
    rng = np.random.default_rng(seed)
    B, S, Hq, Hkv, dh = 2, 7, 4, 2, 8
    q, d_o = rng.standard_normal((2, B, S, Hq, dh))
    k, v = rng.standard_normal((2, B, S, Hkv, dh))
    s, ds = rng.standard_normal((2, B, Hkv, dh, dh))
    return q, k, v, np.array([-0.3, 0.0]), d_o, s, ds


def test_linear_attention_is_the_sum_over_pairs():
    q, k, v, g, _, s, _ = _linear_case(1)
    lengths = [7, 3]
    o, out = otm.linear_attention_fwd(q, k, v, g, 0.5, s, lengths)
    for b, n in enumerate(lengths):
        for h in range(4):
            j = h // 2
            for t in range(n):
                want = sum(np.exp(g[j] * (t - i)) * (q[b, t, h] @ k[b, i, j]) * v[b, i, j] for i in range(t + 1))
                want = 0.5 * (want + np.exp(g[j] * (t + 1)) * q[b, t, h] @ s[b, j])
                assert np.allclose(o[b, t, h], want, rtol=1e-12, atol=1e-13)
        assert not o[b, n:].any()
        for j in range(2):
            want = np.exp(g[j] * n) * s[b, j] + sum(np.exp(g[j] * (n - 1 - i)) * np.outer(k[b, i, j], v[b, i, j]) for i in range(n))
            assert np.allclose(out[b, j], want, rtol=1e-12, atol=1e-13)


def test_linear_attention_in_pieces_is_linear_attention():
    q, k, v, g, _, s, _ = _linear_case(2)
    o, out = otm.linear_attention_fwd(q, k, v, g, 0.5, s)
    o1, mid = otm.linear_attention_fwd(q[:, :3], k[:, :3], v[:, :3], g, 0.5, s)
    o2, end = otm.linear_attention_fwd(q[:, 3:], k[:, 3:], v[:, 3:], g, 0.5, mid)
    assert np.array_equal(np.concatenate((o1, o2), 1), o) and np.array_equal(end, out)
    gone, _ = otm.linear_attention_fwd(q, k, v, np.array([-np.inf, -np.inf]), 1.0, s)       # no memory: (q_t . k_t) v_t
    assert np.allclose(gone[:, :, 0], np.sum(q[:, :, 0] * k[:, :, 0], -1, keepdims=True) * v[:, :, 0])


def test_linear_attention_gradient_against_differences():
    q, k, v, g, d_o, s, ds = _linear_case(3)
    lengths = [7, 3]

    def f(q, k, v, s):
        o, out = otm.linear_attention_fwd(q, k, v, g, 0.5, s, lengths)
        return float(np.sum(o * d_o) + np.sum(out * ds))

    grads = otm.linear_attention_bwd(q, k, v, g, 0.5, d_o, s, ds, lengths)
    rng, args, h = np.random.default_rng(4), (q, k, v, s), 1e-6
    for i, grad in enumerate(grads):
        u = rng.standard_normal(grad.shape)
        plus, minus = (f(*(a + e * u if n == i else a for n, a in enumerate(args))) for e in (h, -h))
        assert np.isclose((plus - minus) / (2 * h), np.sum(grad * u), rtol=1e-7), i
    assert not grads[0][1, 3:].any() and not grads[1][1, 3:].any() and not grads[2][1, 3:].any()
