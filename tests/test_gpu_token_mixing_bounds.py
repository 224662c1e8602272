"""The norm of queries and keys and linear attention write nothing beside their outputs and the workspaces of just the sizes that are asked for: all of them
lie in one allocation, with patterns between them that have to be there afterwards."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

GUARD, PATTERN = 4096, 0xA5


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


class Guarded:
    """Buffers in one allocation, in front of each and behind the last a guard."""

    def __init__(self, **sizes):
        self.spans, at = {}, GUARD
        for n, size in sizes.items():
            self.spans[n] = (at, at + size)
            at += (size + 255) // 256 * 256 + GUARD
        self.mem = torch.full((at,), PATTERN, dtype=torch.uint8, device="cuda")

    def __getitem__(self, n):
        return self.mem[slice(*self.spans[n])]

    def of(self, n, dtype):
        return self[n].view(dtype)

    def check(self, what):
        free = torch.ones(self.mem.numel(), dtype=torch.bool, device="cuda")
        for a, b in self.spans.values():
            free[a:b] = False
        bad = torch.nonzero(free & (self.mem != PATTERN)).flatten()
        assert bad.numel() == 0, f"{what}: {bad.numel()} bytes written beside {[(n, s) for n, s in self.spans.items()]}, the first at {int(bad[0])}"


def _normal(*shape, dtype=torch.bfloat16):
    return torch.randn(shape, device="cuda").to(dtype)


def _lengths(kind, B, S):
    return None if kind is None else torch.tensor([(S * i // max(1, B - 1)) if kind == "ragged" else S for i in range(B)], dtype=torch.int64, device="cuda")


# tokens of one and of many, around the chunks' ends, one segment and many, few rows and more than a launch has workgroups at once
SHAPES = [(1, 1, 1, 1, 32), (1, 1, 32, 8, 128), (3, 63, 6, 2, 64), (1, 65, 3, 1, 128), (2, 129, 5, 5, 32), (4, 257, 4, 2, 64), (1, 1037, 2, 2, 128),
          (1, 2600, 2, 1, 32), (7, 700, 8, 1, 64), (5, 1037, 18, 6, 64), (140, 100, 16, 4, 128), (128, 1100, 3, 1, 32), (160, 300, 8, 8, 64),
          (300, 5, 12, 4, 128), (1, 9000, 4, 4, 128)]


@pytest.mark.parametrize("B,S,Hq,Hkv,dh", SHAPES)
@pytest.mark.parametrize("lengths", [None, "ragged"])
def test_linear_attention(K, B, S, Hq, Hkv, dh, lengths):
    torch.manual_seed(0)
    q, k, v, d_o = (_normal(B, S, h, dh) for h in (Hq, Hkv, Hkv, Hq))
    s, ds = (_normal(B, Hkv, dh, dh, dtype=torch.float32) for _ in range(2))
    log, n, shape = torch.full((Hkv,), -0.05, device="cuda"), _lengths(lengths, B, S), (B, S, Hq, Hkv, dh)
    of_q, of_kv, of_s = B * S * Hq * dh * 2, B * S * Hkv * dh * 2, B * Hkv * dh * dh * 4
    for carry in (False, True):
        state = lambda t: t if carry else None  # noqa: E731
        m = Guarded(o=of_q, ws=K.linear_attention_workspace_bytes(*shape), state=of_s)
        K.linear_attention_forward(q, k, v, log, n, state(s), *shape, 0.1, m.of("o", torch.bfloat16), state(m.of("state", torch.float32)), m["ws"])
        m.check(f"forward, {carry}")
        m = Guarded(dq=of_q, dk=of_kv, ws=K.linear_attention_backward_workspace_bytes(*shape), dv=of_kv, d_state=of_s)
        K.linear_attention_backward(q, k, v, log, n, state(s), d_o, state(ds), *shape, 0.1, m.of("dq", torch.bfloat16), m.of("dk", torch.bfloat16),
                                    m.of("dv", torch.bfloat16), state(m.of("d_state", torch.float32)), m["ws"])
        m.check(f"backward, {carry}")
    m = Guarded(o=of_q // S, state=of_s)
    m.of("state", torch.float32).copy_(s.flatten())
    K.linear_attention_step(*(t[:, 0].contiguous() for t in (q, k, v)), log, n, m.of("state", torch.float32), B, Hq, Hkv, dh, 0.1, m.of("o", torch.bfloat16))
    m.check("step")


@pytest.mark.parametrize("B,S,Hq,Hkv,dh", SHAPES + [(1, 4095, 5, 3, 32), (2, 2049, 7, 1, 128), (4097, 1, 3, 1, 64)])
@pytest.mark.parametrize("lengths", [None, "ragged"])
def test_qk_norm_rope(K, B, S, Hq, Hkv, dh, lengths):
    torch.manual_seed(1)
    q, k, dq, dk = (_normal(B, S, h, dh) for h in (Hq, Hkv, Hq, Hkv))
    g, n, shape = _normal(dh), _lengths(lengths, B, S), (B, S, Hq, Hkv, dh)
    of_q, of_kv = B * S * Hq * dh * 2, B * S * Hkv * dh * 2
    m = Guarded(q=of_q, rstd_q=B * S * Hq * 4, k=of_kv, rstd_k=B * S * Hkv * 4)
    rstd = [m.of("rstd_q", torch.float32), m.of("rstd_k", torch.float32)]
    K.qk_norm_rope_forward(q, k, g, g, None, n, *shape, 1e-5, 1e4, 0, m.of("q", torch.bfloat16), m.of("k", torch.bfloat16), *rstd)
    m.check("forward")
    b = Guarded(dq=of_q, ws=K.qk_norm_rope_backward_workspace_bytes(*shape), dk=of_kv, dgq=2 * dh, dgk=2 * dh)
    K.qk_norm_rope_backward(q, k, g, g, *rstd, dq, dk, None, n, *shape, 1e4, 0, *(b.of(x, torch.bfloat16) for x in ("dq", "dk", "dgq", "dgk")), 0, b["ws"])
    b.check("backward")
    m.check("backward, statistics")
    assert np.isfinite(float(b.of("dgq", torch.bfloat16).float().sum()))
