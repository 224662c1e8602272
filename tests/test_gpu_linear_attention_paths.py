"""Linear attention of many rows, whose work is cut as that of large calls is: several query heads to a workgroup (pairs of them, and an odd one left over), and
sequences in segments of many chunks that a slowly decaying state runs through.  tests/test_linear_attention_plan.py holds on the host which way each case takes.

The batch is a few rows, of different lengths, over and over: the oracle does each once, and the copies have to be the same bits.  Tolerances as in
test_gpu_linear_attention_means: results are off by their rounding to bf16 alone, 1.01 of it in the 2-norm, states by 2e-6.
"""
import numpy as np
import pytest
import torch

from oracle import token_mixing as otm
from synth import inputs as si
from tests.parity import dev_bf16
from tests.test_gpu_linear_attention_means import _close, _inputs, _state_close

pytestmark = pytest.mark.gpu

SLOW = -1.0 / 4096
CASES = [
    # B, S, Hq, Hkv, dh, log_decay, lengths of the rows that repeat, a state comes in
    (64, 130, 16, 4, 128, -0.02, [130, 70], True),           # forward: two parts of two heads; backward: four heads
    (32, 300, 24, 8, 128, -0.02, [300, 0, 129], False),      # parts of two heads and of one; three heads
    (48, 130, 40, 8, 128, -0.02, [130], True),               # parts of three heads and of two; five heads
    (140, 100, 16, 4, 128, -0.02, [100, 40], False),         # forward: four heads
    (128, 1100, 2, 1, 128, SLOW, [1100, 513, 1089], True),   # segments of many chunks
    (128, 2000, 3, 1, 128, 0.0, [2000], False),              # the same, nothing forgotten
    (130, 70, 8, 4, 64, -0.02, [70, 64], False),
    (150, 100, 10, 2, 64, -0.02, [100, 1, 65], True),
    (96, 1500, 5, 1, 64, SLOW, [1500, 900], True),
    (160, 2000, 2, 1, 64, SLOW, [2000, 1], False),
    (64, 200, 20, 4, 32, -0.02, [200, 150], True),
    (140, 70, 8, 4, 32, -0.02, [70, 64, 3], False),
    (128, 1100, 3, 1, 32, SLOW, [1100, 1024], True),
    (200, 3000, 1, 1, 32, SLOW, [3000, 2500], True),
]


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def _case(B, S, Hq, Hkv, dh, decay, lengths, carry, seed):
    """The rows that repeat (bits, states), which of them each row of the batch is, and a maker of the batch."""
    R = len(lengths)
    bits = _inputs(R, S, Hq, Hkv, dh, 0.0, seed)
    rng = np.random.default_rng(seed + 1)
    s, ds = (rng.standard_normal((R, Hkv, dh, dh)).astype(np.float32) * m if carry else None for m in (8, 2))
    which = torch.arange(B, device="cuda") % R
    batch = lambda t: None if t is None else (dev_bf16(t) if t.dtype != np.float32 else torch.from_numpy(t).cuda())[which].contiguous()  # noqa: E731
    log = np.full(Hkv, decay, np.float32)
    return bits, s, ds, log, which, batch, torch.tensor(lengths, device="cuda")[which].contiguous()


def _copies(t, which, R, what):
    for i in range(R):
        rows = t[which == i]
        assert torch.equal(rows.contiguous().view(torch.uint8), rows[:1].expand_as(rows).contiguous().view(torch.uint8)), f"{what}: copies of row {i} differ"


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,decay,lengths,carry", CASES)
def test_forward(K, B, S, Hq, Hkv, dh, decay, lengths, carry):
    bits, s, _, log, which, batch, n = _case(B, S, Hq, Hkv, dh, decay, lengths, carry, S + dh)
    R, scale = len(lengths), dh ** -0.5
    q, k, v = (batch(bits[x]) for x in "qkv")
    o, out = torch.full_like(q, float("nan")), torch.full((B, Hkv, dh, dh), float("nan"), device="cuda")
    K.linear_attention_forward(q, k, v, torch.from_numpy(log).cuda(), n, batch(s), B, S, Hq, Hkv, dh, scale, o, out,
                               torch.empty(K.linear_attention_workspace_bytes(B, S, Hq, Hkv, dh), dtype=torch.uint8, device="cuda"))
    o_ref, s_ref = otm.linear_attention_fwd(*(si.bf16_bits_to_f64(bits[x]) for x in "qkv"), log.astype(np.float64), scale, s, lengths)
    _copies(o, which, R, "o")
    _copies(out, which, R, "state")
    _close(o[:R], o_ref, "o")
    _state_close(out[:R], s_ref, "state")
    assert all(not o[b, m:].any() for b, m in enumerate(lengths))


@pytest.mark.parametrize("B,S,Hq,Hkv,dh,decay,lengths,carry", CASES)
def test_backward(K, B, S, Hq, Hkv, dh, decay, lengths, carry):
    bits, s, ds, log, which, batch, n = _case(B, S, Hq, Hkv, dh, decay, lengths, carry, S + dh + 1)
    R, scale = len(lengths), dh ** -0.5
    q, k, v, d_o = (batch(bits[x]) for x in ("q", "k", "v", "d_o"))
    got = [torch.full_like(t, float("nan")) for t in (q, k, v)] + [torch.full((B, Hkv, dh, dh), float("nan"), device="cuda")]
    K.linear_attention_backward(q, k, v, torch.from_numpy(log).cuda(), n, batch(s), d_o, batch(ds), B, S, Hq, Hkv, dh, scale, *got,
                                torch.empty(K.linear_attention_backward_workspace_bytes(B, S, Hq, Hkv, dh), dtype=torch.uint8, device="cuda"))
    ref = otm.linear_attention_bwd(*(si.bf16_bits_to_f64(bits[x]) for x in "qkv"), log.astype(np.float64), scale, si.bf16_bits_to_f64(bits["d_o"]), s, ds,
                                   lengths)
    for name, t, r in zip(("dq", "dk", "dv", "d_state_in"), got, ref):
        _copies(t, which, R, name)
        (_state_close if name == "d_state_in" else _close)(t[:R], r, name)
        assert name == "d_state_in" or all(not t[b, m:].any() for b, m in enumerate(lengths)), name
