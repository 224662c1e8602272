"""The oracle of the paged cache, of attention over it and of log-probabilities, against other ways to the same numbers (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import decoder_layer as odl
from oracle import generation as og


def test_e4m3_values_and_rounding():
    x = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(og.e4m3_values(), x, equal_nan=True)
    rng = np.random.default_rng(0)
    for scale in (1.0, 1e-3, 37.0, 448.0):
        v = (rng.standard_normal((50, 32)) * scale).astype(np.float32).astype(np.float64)
        code, e = og.quantise(v)
        amax = np.abs(v).max(-1)
        assert np.all(amax <= 448 * 2.0 ** e) and np.all(amax > 448 * 2.0 ** (e - 1.0))
        want = torch.from_numpy((v * 2.0 ** -e[:, None]).astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        assert np.array_equal(code, want)
    assert og.quantise(np.array([[448.0, 1.0]]))[1][0] == 0 and og.quantise(np.array([[448.01, 1.0]]))[1][0] == 1
    assert og.quantise(np.zeros((1, 4)))[1][0] == 0 and np.all(og.quantise(np.zeros((1, 4)))[0] == 0)
    code, e = og.quantise(np.array([[np.inf, 2.0, np.nan, -np.inf]]))
    assert e[0] == -7 and np.isnan(og.dequantise(code, e)[0, [0, 2, 3]]).all() and og.dequantise(code, e)[0, 1] == 2.0


@pytest.mark.parametrize("layout", [0, 1])
def test_rotation_is_the_layers(layout):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((1, 9, 3, 32))
    ref = odl.rope_rotate(x, odl.rope_angles(9, 32, 1e4), layout)
    for p in range(9):
        y = og.rotate(x[0, p], p, 1e4, layout)
        assert np.allclose(np.linalg.norm(y), np.linalg.norm(x[0, p]))
        assert np.allclose(y, ref[0, p])
    # positions add up: R(a) x . R(b) y depends on a - b
    a, b = x[0, 0], x[0, 1]
    assert np.allclose(np.sum(og.rotate(a, 7, 1e4, layout) * og.rotate(b, 3, 1e4, layout)), np.sum(og.rotate(a, 4, 1e4, layout) * b))


def test_attention_is_causal_softmax_attention_whatever_the_pages():
    rng = np.random.default_rng(2)
    b, s, hq, hkv, dh, page = 2, 11, 4, 2, 8, 16
    q, k, v = rng.standard_normal((b, s, hq, dh)), rng.standard_normal((b, s, hkv, dh)), rng.standard_normal((b, s, hkv, dh))
    table = np.array([[2, 9], [0, 9]])
    cache = {"k": np.full((3, hkv, page, dh), np.nan), "v": np.full((3, hkv, page, dh), np.nan), "page_table": table}
    for i in range(b):
        for t in range(s):
            cache["k"][table[i, 0], :, t], cache["v"][table[i, 0], :, t] = k[i, t], v[i, t]
    kk, vv = (torch.from_numpy(x).repeat_interleave(hq // hkv, 2).transpose(1, 2) for x in (k, v))
    ref = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(1, 2), kk, vv, is_causal=True, scale=0.3).transpose(1, 2).numpy()
    o, lse, mag, _ = og.attention(cache, q, None, None, 0.3)
    assert np.allclose(o, ref) and np.all(mag >= np.abs(o) - 1e-12)
    x = 0.3 * np.einsum("bshd,bhtd->bhst", q, kk.numpy())
    x = np.where(np.tril(np.ones((s, s), bool)), x, -np.inf)
    assert np.allclose(lse, np.log(np.exp(x).sum(-1)))
    # the last four tokens behind the seven before them, and padding
    o4, lse4, *_ = og.attention(cache, q[:, 7:], [7, 7], [4, 2], 0.3)
    assert np.allclose(o4[0], o[0, 7:]) and np.allclose(o4[1, :2], o[1, 7:9]) and np.all(o4[1, 2:] == 0)
    assert np.allclose(lse4[0], lse[0, :, 7:]) and np.all(lse4[1, :, 2:] == -np.inf)


def test_logprobs_against_torch_and_its_gradient():
    rng = np.random.default_rng(3)
    T, V, inverse = 5, 40, 0.7
    x = rng.standard_normal((T, V)) * 3
    x[1, 5:] = -np.inf
    targets = np.array([3, 2, -1, 39, 40])
    got = og.logprobs(x, targets, inverse, 4)
    z = torch.from_numpy(x * inverse)
    logp = torch.log_softmax(z, -1)
    for r in (0, 1, 3):
        assert np.isclose(got[0][r], logp[r, targets[r]]) and np.isclose(got[2][r], torch.logsumexp(z[r], 0))
        assert np.isclose(got[1][r], torch.distributions.Categorical(logits=torch.where(z[r].isinf(), -1e9, z[r])).entropy())
        assert np.allclose(got[4][r], logp[r].topk(4).values) and np.array_equal(got[3][r], logp[r].topk(4).indices)
    for r in (2, 4):
        assert got[0][r] == got[1][r] == got[2][r] == 0 and np.all(got[3][r] == -1)
    assert og.logprobs(np.ones((1, 9)), None, 1.0, 3)[3].tolist() == [[0, 1, 2]]      # of equal ones the lower index first
    x[1, 5:] = -4.0
    dl, dh = rng.standard_normal(T), rng.standard_normal(T)
    t = torch.from_numpy(x).requires_grad_()
    logp = torch.log_softmax(t * inverse, -1)
    keep = torch.tensor([True, True, False, True, False])
    chosen = logp.gather(1, torch.tensor([3, 2, 0, 39, 0])[:, None])[:, 0]
    entropy = -(logp.exp() * logp).sum(-1)
    ((chosen * torch.from_numpy(dl) + entropy * torch.from_numpy(dh)) * keep).sum().backward()
    assert np.allclose(og.logprobs_gradient(x, targets, inverse, dl, dh), t.grad.numpy())
    assert np.all(og.logprobs_gradient(np.full((1, 8), -np.inf), [2], 1.0, [1.0], [1.0]) == 0)
