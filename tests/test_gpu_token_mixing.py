"""The norm of queries and keys with the rotary embedding, and linear attention, through the C ABI against the fp64 oracle.

Tolerances, from the arithmetic:
  norm and rotation   one rounding to bf16 (eight significant bits: at most 2^-8 = 3.91e-3 of a value) on top of fp32 arithmetic
                      (1e-5 at most); angles are evaluated in fp64.  3.95e-3 element by element.
  linear attention    the sums over pairs round the weighted scores and the states to bf16 as operands, and the result: three
                      independent roundings of 1.7e-3 rms.  3.5e-3 in the 2-norm; 2.5e-2 element by element is eight of
                      those deviations.
  states              fp32 sums of products that are exact up to fp32: 2e-6 in the 2-norm.
"""
import numpy as np
import pytest
import torch

from oracle import token_mixing as otm
from synth import inputs as si
from tests.parity import dev_bf16, host_f64, rel_err

pytestmark = pytest.mark.gpu

ELEMENT, NORM, LINEAR_ELEMENT, STATE = 3.95e-3, 3.5e-3, 2.5e-2, 2e-6


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def _bits(rng, shape, std=1.0, mean=0.0):
    return si.f32_to_bf16_bits((rng.standard_normal(shape) * std + mean).astype(np.float32))


def _i64(values):
    return None if values is None else torch.tensor(values, dtype=torch.int64, device="cuda")


def _f32(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def _garbage(shape, dtype=torch.bfloat16):
    return torch.full(shape, float("nan"), dtype=dtype, device="cuda")


def _ws(nbytes):
    return torch.full((max(int(nbytes), 256),), 0xFF, dtype=torch.uint8, device="cuda")


def _spoiled(t, lengths, value=float("nan")):
    """A copy of t [B, S, ...] whose padding holds what no result may see."""
    t = t.clone()
    for b, n in enumerate(lengths or []):
        t[b, max(0, n):] = value
    return t


def _norm_err(got, ref):
    return float(np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-300))


def _within(got, ref, element=np.inf, norm=np.inf, what=""):
    got, ref = (host_f64(t) if isinstance(t, torch.Tensor) else t for t in (got, ref))
    e, n = rel_err(got, ref), _norm_err(got, ref)
    assert e <= element and n <= norm, f"{what}: {e:.3e} element by element (at most {element:.3e}), {n:.3e} in the 2-norm (at most {norm:.3e})"


def _same_bits(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


# ------------------------------------------------------------------ norm and rotation
@pytest.mark.parametrize("B,S,Hq,Hkv,dh,base,layout,start,lengths", [
    (1, 1, 1, 1, 32, 1e4, 0, None, None),
    (1, 1, 32, 8, 128, 5e5, 0, [8191], None),                  # a token of one sequence
    (70, 1, 5, 5, 64, 1e4, 1, "spread", None),                 # a token of many
    (2, 128, 4, 4, 32, 1e4, 1, None, None),
    (3, 65, 6, 2, 64, 1e4, 0, [0, 5, 100000], [65, 0, 1]),
    (3, 65, 7, 3, 128, 5e5, 1, None, [-4, 64, 1000]),          # lengths outside 0..seq; 7 heads fill no group of rows
    (2, 1037, 32, 8, 128, 5e5, 0, None, None),
    (1, 4500, 3, 1, 32, 1e4, 0, None, None),                   # more tokens than waves
])
def test_qk_norm_rope(K, B, S, Hq, Hkv, dh, base, layout, start, lengths):
    rng = np.random.default_rng(S + Hq + dh)
    if start == "spread":
        start = [int(x) for x in rng.integers(0, 40000, B)]
    bits = {n: _bits(rng, (B, S, h, dh), 1.28) for n, h in (("q", Hq), ("k", Hkv))}
    dbits = {n: _bits(rng, (B, S, h, dh)) for n, h in (("q", Hq), ("k", Hkv))}
    gbits = {n: _bits(rng, (dh,), 0.1, 1.0) for n in "qk"}
    x = {n: _spoiled(dev_bf16(b), lengths) for n, b in bits.items()}
    dy = {n: _spoiled(dev_bf16(b), lengths, float("inf")) for n, b in dbits.items()}
    g = {n: dev_bf16(b) for n, b in gbits.items()}
    out = {n: _garbage(t.shape) for n, t in x.items()}
    rstd = {n: _garbage(t.shape[:-1], torch.float32) for n, t in x.items()}
    K.qk_norm_rope_forward(x["q"], x["k"], g["q"], g["k"], _i64(start), _i64(lengths), B, S, Hq, Hkv, dh, 1e-5, base, layout, out["q"],
                           out["k"], rstd["q"], rstd["k"])
    dx = {n: _garbage(t.shape) for n, t in x.items()}
    dg = {n: _garbage((dh,)) for n in "qk"}
    ws = _ws(K.qk_norm_rope_backward_workspace_bytes(B, S, Hq, Hkv, dh))
    back = lambda dx, acc: K.qk_norm_rope_backward(  # noqa: E731
        x["q"], x["k"], g["q"], g["k"], rstd["q"], rstd["k"], dy["q"], dy["k"], _i64(start), _i64(lengths), B, S, Hq, Hkv, dh, base, layout,
        dx["q"], dx["k"], dg["q"], dg["k"], acc, ws)
    back(dx, 0)
    once = {n: t.clone() for n, t in dg.items()}
    again = {n: _garbage(t.shape) for n, t in x.items()}
    back(again, 1)
    for n in "qk":
        xr, gr, dr = (si.bf16_bits_to_f64(b[n]) for b in (bits, gbits, dbits))
        y_ref, r_ref = otm.qk_norm_rope_fwd(xr, gr, 1e-5, base, layout, start, lengths)
        _within(out[n], y_ref, ELEMENT, what=n)
        _within(rstd[n], r_ref, 1e-6, what="rstd " + n)
        dx_ref, dg_ref = otm.qk_norm_rope_bwd(xr, gr, r_ref, dr, base, layout, start, lengths)
        _within(dx[n], dx_ref, ELEMENT, what="d" + n)
        _within(once[n], dg_ref, ELEMENT, what="dgamma " + n)
        assert _same_bits([again[n]], [dx[n]]), n
        _within(dg[n], dg_ref + host_f64(once[n]), ELEMENT, what="accumulated dgamma " + n)
    # in place, without statistics; the gradient in place of dy
    y = {n: t.clone() for n, t in x.items()}
    K.qk_norm_rope_forward(y["q"], y["k"], g["q"], g["k"], _i64(start), _i64(lengths), B, S, Hq, Hkv, dh, 1e-5, base, layout, y["q"], y["k"],
                           None, None)
    back(dy, 0)
    for n in "qk":
        assert _same_bits((y[n], dy[n], dg[n]), (out[n], dx[n], once[n])), n


def test_qk_norm_rope_rotation_matches_rope_apply(K):
    """Heads of mean square one and gains of one: the norm gives what went in, and what is left is rope_apply."""
    B, S, H, dh = 2, 384, 3, 64
    rng = np.random.default_rng(5)
    x = dev_bf16(si.f32_to_bf16_bits(np.sign(rng.standard_normal((B, S, H, dh))).astype(np.float32)))   # +-1: mean square 1 exactly
    one = torch.ones(dh, dtype=torch.bfloat16, device="cuda")
    q, k, z = _garbage(x.shape), _garbage(x.shape), x.clone()
    K.qk_norm_rope_forward(x, x, one, one, None, None, B, S, H, H, dh, 0.0, 1e4, 0, q, k, None, None)
    K.rope_apply(z, B, S, H, dh, 1e4, 0, 0)
    assert _same_bits([q], [k])
    # sums of two products in fp32, contracted differently: next to a tie they round to neighbours
    _within(q, host_f64(z), 2 * ELEMENT)
    assert (q != z).float().mean().item() < 1e-3


# ------------------------------------------------------------------ linear attention
SLOW, FAST, MIXED = -1.0 / 4096, -20.0, "mixed"


def _decays(kind, Hkv):
    if kind == "mixed":
        return np.log1p(-np.exp2(-5 - 7 * np.arange(Hkv) / max(1, Hkv - 1))).astype(np.float32)
    return np.full(Hkv, kind, np.float32)


LINEAR_CASES = [
    # B, S, Hq, Hkv, dh, log_decay, state, lengths
    (1, 1, 1, 1, 32, MIXED, True, None),
    (2, 1, 8, 2, 128, MIXED, False, None),
    (1, 63, 2, 2, 64, MIXED, False, None),
    (2, 64, 2, 1, 128, MIXED, True, None),
    (1, 65, 3, 1, 128, MIXED, True, None),
    (3, 128, 6, 2, 32, 0.0, False, None),                      # nothing forgotten
    (3, 129, 6, 2, 64, -np.inf, True, None),                   # nothing remembered
    (1, 200, 4, 4, 128, FAST, True, None),                     # weights that underflow within a chunk
    (4, 257, 4, 2, 64, MIXED, True, [257, 0, 1, 130]),         # a row without a token, and one of one
    (3, 193, 5, 5, 32, MIXED, False, [-3, 64, 9999]),          # lengths outside 0..seq
    (2, 700, 8, 1, 64, SLOW, True, None),                      # eight query heads share one state
    (1, 1037, 2, 2, 128, MIXED, True, [1000]),
    (1, 2600, 2, 1, 32, MIXED, True, None),
    (1, 2305, 1, 1, 128, 0.0, True, None),
]


def _linear_inputs(B, S, Hq, Hkv, dh, decay, carry, seed):
    rng = np.random.default_rng(seed)
    bits = {n: _bits(rng, (B, S, h, dh)) for n, h in (("q", Hq), ("k", Hkv), ("v", Hkv), ("d_o", Hq))}
    s, ds = (rng.standard_normal((B, Hkv, dh, dh)).astype(np.float32) * m if carry else None for m in (4, 1))
    return bits, _decays(decay, Hkv), s, ds


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,decay,carry,lengths", LINEAR_CASES)
def test_linear_attention_forward(K, B, S, Hq, Hkv, dh, decay, carry, lengths):
    bits, log, s, _ = _linear_inputs(B, S, Hq, Hkv, dh, decay, carry, S + dh)
    scale = dh ** -0.5
    q, k, v = (_spoiled(dev_bf16(bits[n]), lengths, x) for n, x in (("q", float("nan")), ("k", float("inf")), ("v", float("nan"))))
    o, out = _garbage(q.shape), _garbage((B, Hkv, dh, dh), torch.float32)
    ws = _ws(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh))
    K.linear_attention_forward(q, k, v, _f32(log), _i64(lengths), _f32(s), B, S, Hq, Hkv, dh, scale, o, out, ws)
    o_ref, s_ref = otm.linear_attention_fwd(*(si.bf16_bits_to_f64(bits[n]) for n in "qkv"), log.astype(np.float64), scale, s, lengths)
    _within(o, o_ref, LINEAR_ELEMENT, NORM, "o")
    _within(out, s_ref, norm=STATE, what="state")
    for b, n in enumerate(lengths or []):
        assert not host_f64(o)[b, max(0, n):].any()
        if s is not None and n <= 0:
            assert torch.equal(out[b], _f32(s)[b])             # a row without a token keeps its state
    # without a state out: the same bits; with the state in place: the same bits again
    o2, o3, io = _garbage(q.shape), _garbage(q.shape), _f32(s if s is not None else np.zeros((B, Hkv, dh, dh)))
    K.linear_attention_forward(q, k, v, _f32(log), _i64(lengths), _f32(s), B, S, Hq, Hkv, dh, scale, o2, None, ws)
    K.linear_attention_forward(q, k, v, _f32(log), _i64(lengths), io, B, S, Hq, Hkv, dh, scale, o3, io, ws)
    assert _same_bits((o, o, io), (o2, o3, out))


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,decay,carry,lengths", LINEAR_CASES)
def test_linear_attention_backward(K, B, S, Hq, Hkv, dh, decay, carry, lengths):
    bits, log, s, ds = _linear_inputs(B, S, Hq, Hkv, dh, decay, carry, S + dh + 1)
    scale = dh ** -0.5
    nan, inf = float("nan"), float("inf")
    q, k, v, d_o = (_spoiled(dev_bf16(bits[n]), lengths, x) for n, x in (("q", nan), ("k", inf), ("v", nan), ("d_o", -inf)))
    ws = _ws(K.linear_attention_backward_workspace_bytes(B, S, Hq, Hkv, dh))

    def run(ds_out, want_state, d_state=None):
        dq, dk, dv = _garbage(q.shape), _garbage(k.shape), _garbage(v.shape)
        d_state = _garbage((B, Hkv, dh, dh), torch.float32) if d_state is None and want_state else d_state
        K.linear_attention_backward(q, k, v, _f32(log), _i64(lengths), _f32(s), d_o, ds_out, B, S, Hq, Hkv, dh, scale, dq, dk, dv, d_state, ws)
        return dq, dk, dv, d_state

    got = run(_f32(ds), True)
    ref = otm.linear_attention_bwd(*(si.bf16_bits_to_f64(bits[n]) for n in "qkv"), log.astype(np.float64), scale,
                                   si.bf16_bits_to_f64(bits["d_o"]), s, ds, lengths)
    for n, a, r in zip(("dq", "dk", "dv"), got, ref):
        _within(a, r, LINEAR_ELEMENT, NORM, n)
        for b, m in enumerate(lengths or []):
            assert not host_f64(a)[b, max(0, m):].any(), n
    _within(got[3], ref[3], norm=STATE, what="d_state_in")
    plain = run(_f32(ds), False)
    io = _f32(ds if ds is not None else np.zeros((B, Hkv, dh, dh)))
    same = run(io, True, io)
    assert _same_bits(got[:3], plain[:3]) and _same_bits(got, same)


@pytest.mark.parametrize("dh,Hq,Hkv,S", [(128, 4, 2, 300), (64, 3, 3, 1000), (32, 2, 1, 150)])
def test_linear_attention_gradient_against_differences(K, dh, Hq, Hkv, S):
    """o is linear in q, in v, and (from no state) in k: a difference over any step is the gradient's product with it."""
    B, scale = 2, dh ** -0.5
    bits, log, _, _ = _linear_inputs(B, S, Hq, Hkv, dh, MIXED, False, 7)
    t = {n: dev_bf16(b) for n, b in bits.items()}
    ws = _ws(max(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh), K.linear_attention_backward_workspace_bytes(B, S, Hq, Hkv, dh)))
    grads = {n: _garbage(t[n].shape) for n in "qkv"}
    K.linear_attention_backward(t["q"], t["k"], t["v"], _f32(log), None, None, t["d_o"], None, B, S, Hq, Hkv, dh, scale, grads["q"],
                                grads["k"], grads["v"], None, ws)
    rng = np.random.default_rng(8)
    d_o = host_f64(t["d_o"])
    for n in "qkv":
        u = dev_bf16(_bits(rng, tuple(t[n].shape)))
        o = _garbage(t["q"].shape)
        args = dict(t, **{n: u})
        K.linear_attention_forward(args["q"], args["k"], args["v"], _f32(log), None, None, B, S, Hq, Hkv, dh, scale, o, None, ws)
        # both sides are sums of N products whose relative errors (NORM) are independent: sqrt(N) of them, six deviations
        left, right = np.sum(host_f64(o) * d_o), np.sum(host_f64(grads[n]) * host_f64(u))
        noise = NORM * (np.linalg.norm(host_f64(o) * d_o) + np.linalg.norm(host_f64(grads[n]) * host_f64(u)))
        assert abs(left - right) <= 6 * noise, n


@pytest.mark.parametrize("B,Hq,Hkv,dh,decay,lengths", [
    (1, 32, 8, 128, MIXED, None), (300, 8, 2, 128, MIXED, None), (7, 5, 5, 64, 0.0, [1, 0, 1, 1, -1, 2, 0]), (3, 9, 3, 32, -np.inf, None),
    (2, 40, 2, 64, MIXED, None),
])
def test_linear_attention_step(K, B, Hq, Hkv, dh, decay, lengths):
    """Three tokens, one after the other, against the oracle; rows without a token stay as they are."""
    bits, log, s, _ = _linear_inputs(B, 3, Hq, Hkv, dh, decay, True, B + dh)
    q, k, v = (dev_bf16(bits[n]) for n in "qkv")
    state, scale = _f32(s), dh ** -0.5
    n = [3 if lengths is None or x > 0 else 0 for x in (lengths or [1] * B)]
    o_ref, s_ref = otm.linear_attention_fwd(*(si.bf16_bits_to_f64(bits[m]) for m in "qkv"), log.astype(np.float64), scale, s, n)
    for t in range(3):
        args = [_spoiled(x[:, t:t + 1].contiguous(), None if lengths is None else [min(1, m) for m in n]) for x in (q, k, v)]
        o = _garbage((B, Hq, dh))
        K.linear_attention_step(*args, _f32(log), _i64(lengths), state, B, Hq, Hkv, dh, scale, o)
        _within(o, o_ref[:, t], ELEMENT, what=f"token {t}")
    _within(state, s_ref, norm=1e-6, what="state")
    for b, m in enumerate(n):
        assert m or torch.equal(state[b], _f32(s)[b])


def test_linear_attention_steps_continue_a_prompt(K):
    B, S, Hq, Hkv, dh = 2, 150, 4, 2, 64
    bits, log, _, _ = _linear_inputs(B, S, Hq, Hkv, dh, MIXED, False, 3)
    q, k, v = (dev_bf16(bits[n]) for n in "qkv")
    ws = _ws(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh))
    whole, end = _garbage(q.shape), _garbage((B, Hkv, dh, dh), torch.float32)
    K.linear_attention_forward(q, k, v, _f32(log), None, None, B, S, Hq, Hkv, dh, 0.125, whole, end, ws)
    cut = 147
    head = [x[:, :cut].contiguous() for x in (q, k, v)]
    o, state = _garbage(head[0].shape), _garbage(end.shape, torch.float32)
    K.linear_attention_forward(*head, _f32(log), None, None, B, cut, Hq, Hkv, dh, 0.125, o, state, ws)
    for t in range(cut, S):
        one = _garbage((B, Hq, dh))
        K.linear_attention_step(*(x[:, t].contiguous() for x in (q, k, v)), _f32(log), None, state, B, Hq, Hkv, dh, 0.125, one)
        _within(one, whole[:, t], norm=2 * NORM, what=f"token {t}")
    _within(state, end, norm=STATE, what="state")


def test_other_streams_and_repeated_calls_give_the_same_bits(K):
    B, S, Hq, Hkv, dh = 2, 515, 6, 2, 64
    bits, log, s, ds = _linear_inputs(B, S, Hq, Hkv, dh, MIXED, True, 9)
    q, k, v, d_o = (dev_bf16(bits[n]) for n in ("q", "k", "v", "d_o"))
    g, s, ds, log = torch.ones(dh, dtype=torch.bfloat16, device="cuda"), _f32(s), _f32(ds), _f32(log)
    n = max(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh), K.linear_attention_backward_workspace_bytes(B, S, Hq, Hkv, dh),
            K.qk_norm_rope_backward_workspace_bytes(B, S, Hq, Hkv, dh))

    def everything(stream):
        """Norm, attention and both gradients, one after the other through one workspace."""
        ws = _ws(n)
        b16 = [_garbage(t.shape) for t in (q, k, q, q, k, v, q, k, g, g)]
        f32 = [_garbage(t.shape, torch.float32) for t in (q[..., 0], k[..., 0], s, s)]
        torch.cuda.synchronize()
        qn, kn, o, dqn, dkn, dv, dq, dk, dgq, dgk = b16
        K.qk_norm_rope_forward(q, k, g, g, None, None, B, S, Hq, Hkv, dh, 1e-5, 1e4, 0, qn, kn, f32[0], f32[1], stream=stream)
        K.linear_attention_forward(qn, kn, v, log, None, s, B, S, Hq, Hkv, dh, 0.125, o, f32[2], ws, stream=stream)
        K.linear_attention_backward(qn, kn, v, log, None, s, d_o, ds, B, S, Hq, Hkv, dh, 0.125, dqn, dkn, dv, f32[3], ws, stream=stream)
        K.qk_norm_rope_backward(q, k, g, g, f32[0], f32[1], dqn, dkn, None, None, B, S, Hq, Hkv, dh, 1e4, 0, dq, dk, dgq, dgk, 0, ws, stream=stream)
        torch.cuda.synchronize()
        return b16 + f32

    first = everything(None)
    for stream in (None, torch.cuda.Stream(), torch.cuda.Stream()):
        assert _same_bits(first, everything(stream))


def test_token_mixing_replays_from_a_hip_graph(K):
    B, S, Hq, Hkv, dh = 1, 700, 4, 2, 128
    bits, log, s, ds = _linear_inputs(B, S, Hq, Hkv, dh, MIXED, True, 10)
    q, k, v, d_o = (dev_bf16(bits[n]) for n in ("q", "k", "v", "d_o"))
    g, s, ds, log = torch.ones(dh, dtype=torch.bfloat16, device="cuda"), _f32(s), _f32(ds), _f32(log)
    ws = _ws(max(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh), K.linear_attention_backward_workspace_bytes(B, S, Hq, Hkv, dh),
                 K.qk_norm_rope_backward_workspace_bytes(B, S, Hq, Hkv, dh)))
    b16 = [_garbage(t.shape) for t in (q, k, q, q, k, v, q, k, g, g)]
    f32 = [_garbage(t.shape, torch.float32) for t in (q[..., 0], k[..., 0], s, s)]
    step = s.clone()

    def work():
        qn, kn, o, dqn, dkn, dv, dq, dk, dgq, dgk = b16
        K.qk_norm_rope_forward(q, k, g, g, None, None, B, S, Hq, Hkv, dh, 1e-5, 1e4, 0, qn, kn, f32[0], f32[1])
        K.linear_attention_forward(qn, kn, v, log, None, s, B, S, Hq, Hkv, dh, 0.125, o, f32[2], ws)
        K.linear_attention_backward(qn, kn, v, log, None, s, d_o, ds, B, S, Hq, Hkv, dh, 0.125, dqn, dkn, dv, f32[3], ws)
        K.qk_norm_rope_backward(q, k, g, g, f32[0], f32[1], dqn, dkn, None, None, B, S, Hq, Hkv, dh, 1e4, 0, dq, dk, dgq, dgk, 0, ws)
        K.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], log, None, step, B, Hq, Hkv, dh, 0.125, o[:, 0])

    work()
    torch.cuda.synchronize()
    want, state = [t.clone() for t in b16 + f32], step.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(3):
        for t in b16 + f32:
            t.fill_(float("nan"))
        step.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert _same_bits(want + [state], b16 + f32 + [step])


def test_bad_arguments_are_rejected_before_any_launch(K):
    B, S, H, dh = 1, 4, 2, 64
    t = torch.zeros((B, S, H, dh), dtype=torch.bfloat16, device="cuda")
    g, log = torch.zeros(dh, dtype=torch.bfloat16, device="cuda"), torch.zeros(H, device="cuda")
    out, state, ws = torch.full_like(t, 7.0), torch.zeros((B, H, dh, dh), device="cuda"), _ws(1 << 20)
    odd = torch.zeros(t.numel() + 8, dtype=torch.bfloat16, device="cuda")[1:1 + t.numel()].view(t.shape)
    fwd = lambda q=t, g=g, S=S, H=H, dh=dh, eps=1e-5, base=1e4, layout=0, rk=None: K.qk_norm_rope_forward(  # noqa: E731
        q, t, g, g, None, None, B, S, H, H, dh, eps, base, layout, out, out, None, rk)
    lin = lambda q=t, log=log, S=S, Hq=H, dh=dh, ws=ws: K.linear_attention_forward(q, t, t, log, None, None, B, S, Hq, H, dh, 1.0, out, None, ws)  # noqa: E731
    step = lambda q=t, state=state, dh=dh: K.linear_attention_step(q, t, t, log, None, state, B, H, H, dh, 1.0, out)  # noqa: E731
    back = lambda ws=ws, d_o=t: K.linear_attention_backward(t, t, t, log, None, None, d_o, None, B, S, H, H, dh, 1.0, out, out, out, None, ws)  # noqa: E731
    norm = lambda rq=log, ws=ws: K.qk_norm_rope_backward(t, t, g, g, rq, log, t, t, None, None, B, S, H, H, dh, 1e4, 0, out, out, g, g, 0, ws)  # noqa: E731
    for call, word in [
        (lambda: fwd(dh=96), "head_dim"), (lambda: fwd(S=0), "non-positive"), (lambda: fwd(H=-1), "non-positive"), (lambda: fwd(q=None), "pointer q"),
        (lambda: fwd(q=odd), "pointer q"), (lambda: fwd(g=None), "gamma_q"), (lambda: fwd(eps=-1.0), "eps"), (lambda: fwd(base=0.0), "rope_base"),
        (lambda: fwd(layout=2), "rope_layout"), (lambda: fwd(rk=log), "go together"), (lambda: norm(rq=None), "rstd"), (lambda: norm(ws=None), "workspace"),
        (lambda: lin(dh=16), "head_dim"), (lambda: lin(Hq=3), "multiple"), (lambda: lin(S=-2), "non-positive"), (lambda: lin(q=odd), "pointer q"),
        (lambda: lin(log=None), "log_decay"), (lambda: lin(ws=None), "workspace"), (lambda: step(state=None), "state"), (lambda: step(dh=48), "head_dim"),
        (lambda: step(q=None), "pointer q"), (lambda: back(ws=None), "workspace"), (lambda: back(d_o=odd), "d_o"),
        (lambda: lin(q=t.cpu()), "GPU"), (lambda: lin(q=t.transpose(1, 2)), "contiguous"),
    ]:
        with pytest.raises(K.DLayerError, match=word):
            call()
    torch.cuda.synchronize()
    assert (out == 7.0).all()
    assert K.linear_attention_workspace_bytes(1, 0, 2, 2, 64) == 0 and K.linear_attention_backward_workspace_bytes(1, 5, 3, 2, 64) == 0
    assert K.qk_norm_rope_backward_workspace_bytes(1, 5, 2, 2, 80) == 0
