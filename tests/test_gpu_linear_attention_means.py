"""Linear attention of inputs that have means, as those of a trained model do: a state is then a large rank-one part and, in front of it, what tells tokens
apart, and a query that is orthogonal to the keys' mean sees the latter alone.  A state rounded to few bits shows here as it does not where all inputs are
independent of mean zero.

Tolerances.  Before a result is rounded to bf16 it is off by what the two-term operands leave: emulated in fp64 with each of those roundings, 2e-6 to 2e-5 of its
2-norm for means of up to four deviations; 1e-4 is allowed.  With the rounding itself, R (that of the oracle's result), independent of it: sqrt(R^2 + 1e-8 |ref|^2),
which is 1.002 R or less.  1.01 R in the 2-norm.  Element by element: half a unit (at most 2^-8 of the value) and six of those 1e-4 deviations.
A state in one fp16 comes to 1.7 R at means of half a deviation and to 5 R at one, a state in one bf16 to 1.3 R without any means.
States: fp32 sums of products exact up to fp32, 2e-6 in the 2-norm.
"""
import numpy as np
import pytest
import torch

from oracle import token_mixing as otm
from synth import inputs as si
from tests.parity import dev_bf16, host_f64, rounded

pytestmark = pytest.mark.gpu

BEFORE_ROUNDING, STATE = 1e-4, 2e-6
SLOW = -1.0 / 4096


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def _means(dh):
    """Two orthogonal vectors of +-1."""
    sign = np.where(np.arange(dh) * 7919 % 31 < 15, 1.0, -1.0)
    return sign, sign * np.where(np.arange(dh) % 2, 1.0, -1.0)


def _around(rng, shape, mean, orthogonal_to):
    """Values of deviation one around `mean`, without what lies along another vector."""
    x = rng.standard_normal(shape)
    u = orthogonal_to / np.linalg.norm(orthogonal_to)
    return si.f32_to_bf16_bits((x - (x @ u)[..., None] * u + mean).astype(np.float32))


def _inputs(B, S, Hq, Hkv, dh, mean, seed):
    """q orthogonal to the keys' mean, k to the queries', v to that of d_o, d_o to that of v."""
    rng, (a, b) = np.random.default_rng(seed), _means(dh)
    return {"q": _around(rng, (B, S, Hq, dh), mean * a, b), "k": _around(rng, (B, S, Hkv, dh), mean * b, a),
            "v": _around(rng, (B, S, Hkv, dh), mean * a, b), "d_o": _around(rng, (B, S, Hq, dh), mean * b, a)}


def _close(got, ref, what):
    got, size = host_f64(got), np.linalg.norm(ref)
    assert np.all(np.isfinite(got)), what
    rounding, off = np.linalg.norm(rounded(ref) - ref), np.linalg.norm(got - ref)
    assert off <= 1.01 * rounding, f"{what}: {off / size:.3e} in the 2-norm, its rounding is {rounding / size:.3e}"
    bound = 2.0 ** -8 * np.abs(ref) + 6 * BEFORE_ROUNDING * size / np.sqrt(ref.size)
    worst = np.max(np.abs(got - ref) / np.maximum(bound, 1e-300))
    assert worst <= 1.0, f"{what}: an element is off by {worst:.2f} times its bound"


def _state_close(got, ref, what):
    got = got.double().cpu().numpy()
    assert np.linalg.norm(got - ref) <= STATE * np.linalg.norm(ref), what


CASES = [
    # B, S, Hq, Hkv, dh, mean / deviation, log_decay, a state comes in
    (1, 2100, 2, 1, 128, 1.0, SLOW, False),
    (1, 2100, 1, 1, 128, 4.0, SLOW, True),
    (1, 1500, 3, 1, 128, 0.5, 0.0, False),
    (2, 1100, 4, 2, 64, 1.0, SLOW, True),
    (1, 4000, 1, 1, 64, 2.0, SLOW, False),
    (1, 3000, 2, 1, 32, 1.0, SLOW, False),
    (2, 40, 5, 1, 128, 2.0, SLOW, True),        # fewer tokens than a chunk: the state that comes in alone
    (3, 64, 2, 2, 32, 2.0, SLOW, True),
]


def _states(rng, B, Hkv, dh, mean, tokens, along_rows, along_columns):
    """What so many tokens leave: their common part, and their deviations."""
    return (tokens * mean ** 2 * np.outer(along_rows, along_columns) + np.sqrt(tokens) * rng.standard_normal((B, Hkv, dh, dh))).astype(np.float32)


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,mean,decay,carry", CASES)
def test_forward(K, B, S, Hq, Hkv, dh, mean, decay, carry):
    bits, (a, b) = _inputs(B, S, Hq, Hkv, dh, mean, S + dh), _means(dh)
    s = _states(np.random.default_rng(dh), B, Hkv, dh, mean, 4096, b, a) if carry else None
    log, scale = np.full(Hkv, decay, np.float32), dh ** -0.5
    q, k, v = (dev_bf16(bits[n]) for n in "qkv")
    o, out = torch.full_like(q, float("nan")), torch.full((B, Hkv, dh, dh), float("nan"), device="cuda")
    K.linear_attention_forward(q, k, v, torch.from_numpy(log).cuda(), None, None if s is None else torch.from_numpy(s).cuda(), B, S, Hq, Hkv, dh, scale,
                               o, out, torch.empty(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh), dtype=torch.uint8, device="cuda"))
    o_ref, s_ref = otm.linear_attention_fwd(*(si.bf16_bits_to_f64(bits[n]) for n in "qkv"), log.astype(np.float64), scale, s)
    _close(o, o_ref, "o")
    _state_close(out, s_ref, "state")


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,mean,decay,carry", CASES)
def test_backward(K, B, S, Hq, Hkv, dh, mean, decay, carry):
    bits, (a, b) = _inputs(B, S, Hq, Hkv, dh, mean, S + dh + 1), _means(dh)
    rng, scale = np.random.default_rng(dh), dh ** -0.5
    s = _states(rng, B, Hkv, dh, mean, 4096, b, a) if carry else None
    ds = _states(rng, B, Hkv, dh, mean, 4096 * scale, a, b) if carry else None
    log = np.full(Hkv, decay, np.float32)
    q, k, v, d_o = (dev_bf16(bits[n]) for n in ("q", "k", "v", "d_o"))
    dev = lambda x: None if x is None else torch.from_numpy(x).cuda()  # noqa: E731
    grads, d_state = [torch.full_like(t, float("nan")) for t in (q, k, v)], torch.full((B, Hkv, dh, dh), float("nan"), device="cuda")
    K.linear_attention_backward(q, k, v, dev(log), None, dev(s), d_o, dev(ds), B, S, Hq, Hkv, dh, scale, *grads, d_state,
                                torch.empty(K.linear_attention_backward_workspace_bytes(B, S, Hq, Hkv, dh), dtype=torch.uint8, device="cuda"))
    ref = otm.linear_attention_bwd(*(si.bf16_bits_to_f64(bits[n]) for n in "qkv"), log.astype(np.float64), scale, si.bf16_bits_to_f64(bits["d_o"]), s, ds)
    for n, g, r in zip(("dq", "dk", "dv"), grads, ref):
        _close(g, r, n)
    _state_close(d_state, ref[3], "d_state_in")


@pytest.mark.parametrize("dh,mean", [(32, 1.0), (64, 1.0), (128, 2.0)])
def test_columns_of_different_size(K, dh, mean):
    """Values whose columns' sizes span 2^16: every column of o is right by itself (o = S^T q keeps them apart), although the state meets queries scaled as a whole."""
    B, S, Hq, Hkv = 1, 1500, 2, 1
    bits = _inputs(B, S, Hq, Hkv, dh, mean, dh + 5)
    size = 2.0 ** -(np.arange(dh) * 16 // (dh - 1))
    bits["v"] = si.f32_to_bf16_bits((si.bf16_bits_to_f64(bits["v"]) * size).astype(np.float32))   # exact
    q, k, v = (dev_bf16(bits[n]) for n in "qkv")
    log, o, scale = np.full(Hkv, SLOW, np.float32), torch.empty_like(q), dh ** -0.5
    K.linear_attention_forward(q, k, v, torch.from_numpy(log).cuda(), None, None, B, S, Hq, Hkv, dh, scale, o, None,
                               torch.empty(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh), dtype=torch.uint8, device="cuda"))
    o_ref, _ = otm.linear_attention_fwd(*(si.bf16_bits_to_f64(bits[n]) for n in "qkv"), log.astype(np.float64), scale)
    for c in range(dh):
        _close(o[..., c], o_ref[..., c], f"column {c}, of size {size[c]}")


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_an_infinite_element_of_a_state_stays_in_its_column(K, dh):
    B, S, Hq, Hkv = 1, 100, 2, 1
    bits = _inputs(B, S, Hq, Hkv, dh, 0.0, dh)
    q, k, v = (dev_bf16(bits[n]) for n in "qkv")
    s = torch.from_numpy(np.random.default_rng(3).standard_normal((B, Hkv, dh, dh)).astype(np.float32)).cuda()
    log, ws = torch.full((Hkv,), -0.01, device="cuda"), torch.empty(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh), dtype=torch.uint8, device="cuda")
    row, col, out = 5, 17, []
    for x in (0.0, float("inf")):
        s[0, 0, row, col] = x
        out.append(torch.empty_like(q))
        K.linear_attention_forward(q, k, v, log, None, s, B, S, Hq, Hkv, dh, dh ** -0.5, out[-1], None, ws)
    others = torch.arange(dh, device="cuda") != col
    assert torch.equal(out[0][..., others], out[1][..., others])
    # lambda^(t+1) q_t[row] times infinity: of q's sign
    assert torch.equal(out[1][..., col].float(), q[..., row].float().sign() * float("inf"))
