"""Norms and rotation of queries and keys, and linear attention with a decay for each head: the calls that these operators' performance
is judged on, at the sizes their users run, with the operators' plain form in elementary torch operations.

Kinds of cases
  qk_norm  qk_norm_rope_forward (direction "forward": with the statistics a training step keeps; "decode": one token a row, each at a
           position of its own, no statistics) or qk_norm_rope_backward ("backward")
  linear   linear_attention_forward ("forward"), linear_attention_backward ("backward"), or linear_attention_step ("step": one token
           a row, the state updated in place)

lengths: "full", or "ragged": row i of a batch holds about i / (batch - 1) of seq tokens (the first none, the last all), the rest is padding.
carry: a state comes in with the call and goes out of it (and their gradients in the backward).
"""
import math

import torch

own = False

EPS = 1e-5
CHUNK = 64               # tokens of a chunk of the plain form


# ------------------------------------------------------------------ the cases
def _qk(direction, batch, seq, n_q_heads, n_kv_heads, head_dim, rope_base=1e4, rope_layout=0, lengths="full", name=None):
    c = dict(kind="qk_norm", direction=direction, batch=batch, seq=seq, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
             rope_base=rope_base, rope_layout=rope_layout, lengths=lengths)
    return dict(c, name=name) if name else c


def _linear(direction, batch, seq, n_q_heads, n_kv_heads, head_dim, lengths="full", carry=False, name=None):
    c = dict(kind="linear", direction=direction, batch=batch, seq=seq, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim,
             lengths=lengths, carry=carry)
    return dict(c, name=name) if name else c


def listed():
    return [
        # generating one sequence with an 8B-shaped model: one token's heads, nothing but latency
        _qk("decode", 1, 1, 32, 8, 128, rope_base=5e5, name="qk_decode_1"),
        # generating many sequences at once
        _qk("decode", 256, 1, 32, 8, 128, rope_base=5e5, name="qk_decode_256"),
        # a training step of the 8B-shaped layer, its two passes
        _qk("forward", 2, 8192, 32, 8, 128, rope_base=5e5, name="qk_8b"),
        _qk("backward", 2, 8192, 32, 8, 128, rope_base=5e5, name="qk_8b_grad"),
        # fine-tuning on texts of different lengths, one of them empty: heads of 64, adjacent pairs, odd sizes
        _qk("backward", 5, 1037, 18, 6, 64, rope_layout=1, lengths="ragged", name="qk_ragged_grad"),
        # generating one sequence, and many, with an 8B-shaped model
        _linear("step", 1, 1, 32, 8, 128, carry=True, name="step_1"),
        _linear("step", 256, 1, 32, 8, 128, carry=True, name="step_256"),
        # a training step of the 8B-shaped layer, its two passes
        _linear("forward", 2, 8192, 32, 8, 128, name="linear_8b"),
        _linear("backward", 2, 8192, 32, 8, 128, name="linear_8b_grad"),
        # the small model's layer, heads of 64 that share nothing
        _linear("backward", 8, 1024, 12, 12, 64, name="linear_small_grad"),
        # training over consecutive pieces of texts of different lengths, the state carried from piece to piece
        _linear("backward", 5, 1037, 18, 6, 32, lengths="ragged", carry=True, name="linear_ragged_grad"),
        # reading one very long prompt before generating from it
        _linear("forward", 1, 65536, 16, 8, 128, carry=True, name="linear_prompt"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    largest = max(_cost(c) for c in listed())
    while True:
        head_dim = rng.choice((32, 64, 64, 128, 128, 128))
        n_kv_heads = _log_int(rng, 1, 16)
        n_q_heads = n_kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
        if n_q_heads * head_dim > 4096:
            continue
        if rng.random() < 0.4:
            direction = rng.choice(("forward", "backward", "backward", "decode"))
            c = _qk(direction, _log_int(rng, 1, 512) if direction == "decode" else rng.randint(1, 8),
                    1 if direction == "decode" else _log_int(rng, 1, 16384), n_q_heads, n_kv_heads, head_dim, rng.choice((1e4, 5e5)),
                    rng.choice((0, 0, 1)), "full" if direction == "decode" else rng.choice(("full", "full", "ragged")))
        else:
            direction = rng.choice(("forward", "forward", "backward", "backward", "step"))
            c = _linear(direction, _log_int(rng, 1, 512) if direction == "step" else rng.randint(1, 8),
                        1 if direction == "step" else _log_int(rng, 1, 65536), n_q_heads, n_kv_heads, head_dim,
                        "full" if direction == "step" else rng.choice(("full", "full", "ragged")), direction == "step" or rng.random() < 0.4)
        if c["lengths"] == "ragged" and c["batch"] == 1:
            continue
        if 3072 not in (c["seq"], n_q_heads * head_dim, n_kv_heads * head_dim) and _cost(c) <= largest:
            return c


def _cost(c):
    """Bytes and operations on one scale, of the padded sizes: what a drawn case is held to."""
    w = work(dict(c, lengths="full"))
    return w["bytes"] + w["flops"] / 50


# ------------------------------------------------------------------ inputs
def _lengths(c):
    """The lengths of a ragged batch (from the case alone, so that its work is known), or None."""
    if c["lengths"] == "full":
        return None
    return [c["seq"] * i // (c["batch"] - 1) for i in range(c["batch"])]


def prepare(case, seed):
    c = case
    b, s, hq, hkv, dh = c["batch"], c["seq"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=gen).to(dtype)

    st = {"case": c}
    lengths = _lengths(c)
    st["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int64, device="cuda")
    if c["kind"] == "qk_norm":
        # projections of normalised tokens by weights of std 0.02 at a width of 4096 have std 1.28
        st["q"], st["k"] = normal(b, s, hq, dh, std=1.28), normal(b, s, hkv, dh, std=1.28)
        st["gamma_q"], st["gamma_k"] = normal(dh, std=0.02, mean=1.0), normal(dh, std=0.02, mean=1.0)
        st["start"] = torch.randint(0, 32768, (b,), generator=gen, device="cuda") if c["direction"] == "decode" else None
        if c["direction"] == "backward":
            st["dq_out"], st["dk_out"] = normal(b, s, hq, dh), normal(b, s, hkv, dh)
            # what the forward left; padding has no statistics
            st["rstd_q"], st["rstd_k"] = ((x.float().square().mean(-1) + EPS).rsqrt() * _valid(st, s)[..., None] for x in (st["q"], st["k"]))
    else:
        # queries and keys as qk_norm_rope leaves them: mean square one
        st["q"], st["k"], st["v"] = normal(b, s, hq, dh), normal(b, s, hkv, dh), normal(b, s, hkv, dh)
        # a head's memory: 1 / (1 - decay) = 2^5 tokens for the first, up to 2^12 for the last
        st["log_decay"] = torch.log1p(-torch.exp2(-5 - 7 * torch.arange(hkv, dtype=torch.float32, device="cuda") / max(1, hkv - 1)))
        st["scale"] = dh ** -0.5
        st["state_in"] = normal(b, hkv, dh, dh, std=4.0, dtype=torch.float32) if c["carry"] else None
        if c["direction"] == "backward":
            st["d_o"] = normal(b, s, hq, dh)
            st["d_state_out"] = normal(b, hkv, dh, dh, dtype=torch.float32) if c["carry"] else None
    return st


def _valid(st, seq):
    """[batch, seq] in 32 bits: 1 for a token, 0 for padding."""
    t = torch.arange(seq, device="cuda")
    n = st["lengths"]
    return torch.ones((st["case"]["batch"], seq), device="cuda") if n is None else (t < n[:, None]).float()


# ------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if own:
        return _own_qk(state, c) if c["kind"] == "qk_norm" else _own_linear(state, c)
    if c["kind"] == "qk_norm":
        return _plain_qk_backward(state, c) if c["direction"] == "backward" else _plain_qk_forward(state, c)
    return {"forward": _plain_linear_forward, "backward": _plain_linear_backward, "step": _plain_linear_step}[c["direction"]](state, c)


def _own_qk(st, c):
    import paper_2602_08387_amd as K
    b, s, hq, hkv, dh = c["batch"], c["seq"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    if "out" not in st:          # a program's own output buffers and workspace, kept from step to step
        if c["direction"] == "backward":
            st["out"] = [torch.empty_like(st[n]) for n in ("q", "k", "gamma_q", "gamma_k")]
            st["ws"] = torch.empty(K.qk_norm_rope_backward_workspace_bytes(b, s, hq, hkv, dh), dtype=torch.uint8, device="cuda")
        else:
            st["out"] = [torch.empty_like(st["q"]), torch.empty_like(st["k"])]
            if c["direction"] == "forward":
                st["out"] += [torch.empty((b, s, h), dtype=torch.float32, device="cuda") for h in (hq, hkv)]
    if c["direction"] == "backward":
        K.qk_norm_rope_backward(st["q"], st["k"], st["gamma_q"], st["gamma_k"], st["rstd_q"], st["rstd_k"], st["dq_out"], st["dk_out"],
                                st["start"], st["lengths"], b, s, hq, hkv, dh, c["rope_base"], c["rope_layout"], *st["out"], 0, st["ws"])
    else:
        q_out, k_out, rstd_q, rstd_k = (st["out"] + [None, None])[:4]
        K.qk_norm_rope_forward(st["q"], st["k"], st["gamma_q"], st["gamma_k"], st["start"], st["lengths"], b, s, hq, hkv, dh, EPS,
                               c["rope_base"], c["rope_layout"], q_out, k_out, rstd_q, rstd_k)
    return st["out"]


def _own_linear(st, c):
    import paper_2602_08387_amd as K
    b, s, hq, hkv, dh = c["batch"], c["seq"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    empty_state = lambda: torch.empty((b, hkv, dh, dh), dtype=torch.float32, device="cuda") if c["carry"] else None  # noqa: E731
    if c["direction"] == "step":
        if "out" not in st:
            st["out"] = [torch.empty_like(st["q"]), st["state_in"]]
        K.linear_attention_step(st["q"], st["k"], st["v"], st["log_decay"], None, st["state_in"], b, hq, hkv, dh, st["scale"], st["out"][0])
        return st["out"]
    if c["direction"] == "forward":
        if "out" not in st:
            st["out"] = [torch.empty_like(st["q"]), empty_state()]
            st["ws"] = torch.empty(K.linear_attention_workspace_bytes(b, s, hq, hkv, dh), dtype=torch.uint8, device="cuda")
        K.linear_attention_forward(st["q"], st["k"], st["v"], st["log_decay"], st["lengths"], st["state_in"], b, s, hq, hkv, dh, st["scale"],
                                   st["out"][0], st["out"][1], st["ws"])
        return st["out"]
    if "out" not in st:
        st["out"] = [torch.empty_like(st[n]) for n in ("q", "k", "v")] + [empty_state()]
        st["ws"] = torch.empty(K.linear_attention_backward_workspace_bytes(b, s, hq, hkv, dh), dtype=torch.uint8, device="cuda")
    K.linear_attention_backward(st["q"], st["k"], st["v"], st["log_decay"], st["lengths"], st["state_in"], st["d_o"], st["d_state_out"],
                                b, s, hq, hkv, dh, st["scale"], *st["out"], st["ws"])
    return st["out"]


# ------------------------------------------------------------------ the plain form: norm and rotation
def _plain_angles(st, c):
    """cos and sin [batch or 1, seq, 1, head_dim / 2] of the tokens' angles."""
    theta = c["rope_base"] ** (-2.0 * torch.arange(c["head_dim"] // 2, dtype=torch.float32, device="cuda") / c["head_dim"])
    p = torch.arange(c["seq"], device="cuda")[None] + (0 if st["start"] is None else st["start"][:, None])
    phi = p.float()[..., None, None] * theta
    return phi.cos(), phi.sin()


def _halves(x, layout):
    return (x[..., 0::2], x[..., 1::2]) if layout else x.chunk(2, -1)


def _joined(a, b, layout):
    return torch.stack((a, b), -1).flatten(-2) if layout else torch.cat((a, b), -1)


def _plain_qk_forward(st, c):
    cos, sin = _plain_angles(st, c)
    valid = (_valid(st, c["seq"]) > 0)[..., None]

    def one(x, gamma):
        x = torch.where(valid[..., None], x.float(), 0.0)
        rstd = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        a, b = _halves(x * rstd * gamma.float(), c["rope_layout"])
        return _joined(a * cos - b * sin, b * cos + a * sin, c["rope_layout"]).bfloat16(), torch.where(valid, rstd[..., 0], 0.0)

    (q_out, rstd_q), (k_out, rstd_k) = one(st["q"], st["gamma_q"]), one(st["k"], st["gamma_k"])
    return [q_out, k_out] if c["direction"] == "decode" else [q_out, k_out, rstd_q, rstd_k]


def _plain_qk_backward(st, c):
    cos, sin = _plain_angles(st, c)
    valid = (_valid(st, c["seq"]) > 0)[..., None, None]

    def one(x, gamma, rstd, dy):
        a, b = _halves(torch.where(valid, dy.float(), 0.0), c["rope_layout"])
        dz = _joined(a * cos + b * sin, b * cos - a * sin, c["rope_layout"])
        xhat = torch.where(valid, x.float(), 0.0) * rstd[..., None]
        dxhat = dz * gamma.float()
        dx = rstd[..., None] * (dxhat - xhat * (dxhat * xhat).mean(-1, keepdim=True))
        return dx.bfloat16(), (dz * xhat).sum((0, 1, 2)).bfloat16()

    dq, dgamma_q = one(st["q"], st["gamma_q"], st["rstd_q"], st["dq_out"])
    dk, dgamma_k = one(st["k"], st["gamma_k"], st["rstd_k"], st["dk_out"])
    return [dq, dk, dgamma_q, dgamma_k]


# ------------------------------------------------------------------ the plain form: linear attention
# Chunks of CHUNK tokens: within one the masked products of queries and keys, from one to the next the states. A query head's rows of a
# chunk are stacked under those of the other heads of its group: [batch, kv head, chunk, group * CHUNK, head_dim].
def _chunked(st, c, name):
    """[batch, kv head, chunk, rows, head_dim] in 32 bits, padding as zeros."""
    b, s, hkv, dh = c["batch"], c["seq"], c["n_kv_heads"], c["head_dim"]
    x = torch.where((_valid(st, s) > 0)[..., None, None], st[name].float(), 0.0)
    g = x.shape[2] // hkv
    x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, -s % CHUNK))
    return x.view(b, -1, CHUNK, hkv, g, dh).permute(0, 3, 1, 4, 2, 5).reshape(b, hkv, -1, g * CHUNK, dh)


def _tokens(x, c):
    """_chunked's way back: [batch, seq, heads, head_dim]."""
    b, hkv, n, rows, dh = x.shape
    return x.view(b, hkv, n, rows // CHUNK, CHUNK, dh).permute(0, 2, 4, 1, 3, 5).reshape(b, n * CHUNK, -1, dh)[:, :c["seq"]]


def _powers(st, c):
    """Decays as products want them: (in a chunk [hkv, 1, group * CHUNK, CHUNK], from the chunk's start to after token i [hkv, 1, rows, 1],
    from after token j to its end [hkv, 1, CHUNK, 1], from one chunk to the next [hkv, chunks, chunks], from the start to chunk [hkv, chunks])."""
    g, n = c["n_q_heads"] // c["n_kv_heads"], -(-c["seq"] // CHUNK)
    log, i, m = st["log_decay"][:, None, None], torch.arange(CHUNK, device="cuda"), torch.arange(n, device="cuda")
    inside = torch.tril(torch.exp(log * (i[:, None] - i[None]).clamp(min=0))).repeat(1, g, 1)
    across = torch.tril(torch.exp(log * CHUNK * (m[:, None] - m[None] - 1).clamp(min=0)), -1)
    return (inside[:, None], torch.exp(log * (i + 1)).repeat(1, 1, g)[..., None], torch.exp(log * (CHUNK - 1 - i))[..., None], across,
            torch.exp(log[..., 0] * CHUNK * m))


def _to_the_end(st, c):
    """[batch, seq, hkv, 1]: the decay from after token t to the end of its row, zero for padding; and [batch, hkv, 1, 1]: of the whole row."""
    s, log = c["seq"], st["log_decay"]
    n = torch.full((c["batch"],), s, device="cuda") if st["lengths"] is None else st["lengths"]
    left = n[:, None] - 1 - torch.arange(s, device="cuda")
    w = torch.where(left[..., None] >= 0, torch.exp(log * left.clamp(min=0)[..., None]), 0.0)
    return w[..., None], torch.exp(log * n[:, None])[..., None, None]


def _chunk_states(st, c, k, v, to_end, across, from_start):
    """[batch, kv head, chunk, head_dim, head_dim]: the state each chunk begins with."""
    u = (k * to_end).transpose(-1, -2) @ v
    h = (across @ u.flatten(-2)).view(u.shape)
    return h if st["state_in"] is None else h + from_start[..., None, None] * st["state_in"][:, :, None]


def _plain_linear_forward(st, c):
    q, k, v = (_chunked(st, c, n) for n in ("q", "k", "v"))
    inside, after, to_end, across, from_start = _powers(st, c)
    h = _chunk_states(st, c, k, v, to_end, across, from_start)
    o = (q @ k.transpose(-1, -2) * inside) @ v + after * (q @ h)
    out = [(_tokens(o, c) * st["scale"]).bfloat16()]
    if not c["carry"]:
        return out + [None]
    w, whole = _to_the_end(st, c)
    valid = (_valid(st, c["seq"]) > 0)[..., None, None]
    kw, vv = (torch.where(valid, st[n].float(), 0.0) for n in ("k", "v"))
    return out + [(kw * w).permute(0, 2, 3, 1) @ vv.permute(0, 2, 1, 3) + whole * st["state_in"]]


def _plain_linear_backward(st, c):
    q, k, v, d_o = (_chunked(st, c, n) for n in ("q", "k", "v", "d_o"))
    d_o = d_o * st["scale"]
    inside, after, to_end, across, from_start = _powers(st, c)
    h = _chunk_states(st, c, k, v, to_end, across, from_start)
    dp = d_o @ v.transpose(-1, -2) * inside
    dq = dp @ k + after * (d_o @ h.transpose(-1, -2))
    w = (q * after).transpose(-1, -2) @ d_o                                    # a chunk's part of the gradient of the state before it
    r = (across.transpose(-1, -2) @ w.flatten(-2)).view(w.shape)               # gradient of the state each chunk ends with
    p = q @ k.transpose(-1, -2) * inside
    dk = _tokens(dp.transpose(-1, -2) @ q + to_end * (v @ r.transpose(-1, -2)), c)
    dv = _tokens(p.transpose(-1, -2) @ d_o + to_end * (k @ r), c)
    if not c["carry"]:
        return [_tokens(dq, c).bfloat16(), dk.bfloat16(), dv.bfloat16(), None]
    left, whole = _to_the_end(st, c)
    valid = (_valid(st, c["seq"]) > 0)[..., None, None]
    kk, vv = (torch.where(valid, st[n].float(), 0.0) for n in ("k", "v"))
    dk = dk + ((vv * left).permute(0, 2, 1, 3) @ st["d_state_out"].transpose(-1, -2)).permute(0, 2, 1, 3)
    dv = dv + ((kk * left).permute(0, 2, 1, 3) @ st["d_state_out"]).permute(0, 2, 1, 3)
    d_state_in = (from_start[..., None, None] * w).sum(2) + whole * st["d_state_out"]
    return [_tokens(dq, c).bfloat16(), dk.bfloat16(), dv.bfloat16(), d_state_in]


def _plain_linear_step(st, c):
    b, hkv, dh = c["batch"], c["n_kv_heads"], c["head_dim"]
    k, v = st["k"].view(b, hkv, dh).float(), st["v"].view(b, hkv, dh).float()
    s = st["state_in"]
    s.mul_(st["log_decay"].exp()[:, None, None]).add_(k[..., None] * v[..., None, :])
    o = st["q"].view(b, hkv, -1, dh).float() @ s * st["scale"]
    return [o.bfloat16().view(st["q"].shape), s]


# ------------------------------------------------------------------ what cannot be done without
def work(case):
    c = case
    hq, hkv, dh = c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    padded, lengths = c["batch"] * c["seq"], _lengths(c)
    tokens = padded if lengths is None else sum(lengths)
    if c["kind"] == "qk_norm":
        row = (hq + hkv) * dh
        read = {"forward": 2, "decode": 2, "backward": 4}[c["direction"]] * row * tokens
        stats = {"forward": 4 * padded, "decode": 0, "backward": 4 * tokens}[c["direction"]] * (hq + hkv)
        return {"bytes": read + 2 * row * padded + stats, "flops": (20 if c["direction"] == "backward" else 9) * row * tokens}
    states = 4 * c["batch"] * hkv * dh * dh
    if c["direction"] == "backward":
        return {"bytes": 2 * dh * (tokens * (2 * hq + 2 * hkv) + padded * (hq + 2 * hkv)) + (3 if c["carry"] else 0) * states,
                "flops": 2 * dh * dh * (2 * hq + 3 * hkv) * tokens}
    return {"bytes": 2 * dh * (tokens * (hq + 2 * hkv) + padded * hq) + (2 if c["carry"] else 0) * states, "flops": 2 * dh * dh * (hq + hkv) * tokens}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    c, st = case, prepare(case, seed)
    rows = [c["seq"]] * c["batch"] if _lengths(c) is None else _lengths(c)
    n_q_heads, n_kv_heads, dh = c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    f64 = dict(dtype=torch.float64, device="cuda")
    back = c["direction"] == "backward"

    def norm_and_rotation(x, gamma, dy):
        """Pairs as complex numbers, one batch row after the other; gradients by torch's differentiation of the definition."""
        theta = c["rope_base"] ** (-2.0 * torch.arange(dh // 2, **f64) / dh)
        gamma = gamma.double().requires_grad_(back)
        out, stat, gain = torch.zeros(x.shape, **f64), torch.zeros(x.shape[:-1], **f64), torch.zeros(dh, **f64)
        for b, n in enumerate(rows):
            p = torch.arange(n, **f64) + (0 if st["start"] is None else int(st["start"][b]))
            turn = torch.polar(torch.ones((), **f64), p[:, None, None] * theta)
            xb = x[b, :n].double().requires_grad_(back)
            rstd = 1 / (xb.pow(2).sum(-1) / dh + EPS).sqrt()
            z = xb * rstd[..., None] * gamma
            z = z.unflatten(-1, (-1, 2)) if c["rope_layout"] else z.unflatten(-1, (2, -1)).transpose(-1, -2)
            y = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            y = (y if c["rope_layout"] else y.transpose(-1, -2)).flatten(-2)
            if back:
                out[b, :n], g = torch.autograd.grad((y * dy[b, :n].double()).sum(), (xb, gamma))
                gain += g
            else:
                out[b, :n], stat[b, :n] = y, rstd
        return out, gain if back else stat

    if c["kind"] == "qk_norm":
        (dq, sq), (dk, sk) = (norm_and_rotation(st[n], st["gamma_" + n], st.get("d%s_out" % n)) for n in ("q", "k"))
        return [dq, dk] if c["direction"] == "decode" else [dq, dk, sq, sk]

    # linear attention: the sums over all pairs s <= t, one batch row and KV head after the other, 2048 queries at a time
    group, scale = n_q_heads // n_kv_heads, st["scale"]
    o, dk, dv = (torch.zeros(st[n].shape, **f64) for n in ("q", "k", "v"))      # o: dq in the backward
    state = torch.zeros(st["state_in"].shape, **f64) if c["carry"] else None    # or its gradient
    for b, n in enumerate(rows):
        for j in range(n_kv_heads):
            log = st["log_decay"][j].double()
            k, v = st["k"][b, :n, j].double(), st["v"][b, :n, j].double()
            s0 = st["state_in"][b, j].double() if c["carry"] else torch.zeros((dh, dh), **f64)
            since = torch.exp(log * (torch.arange(n, **f64) + 1))[:, None]
            left = torch.exp(log * (n - 1 - torch.arange(n, **f64)))[:, None]
            power = torch.exp(log * torch.arange(n, **f64))
            for t0 in range(0, n, 2048):
                t1 = min(n, t0 + 2048)
                gap = torch.arange(t0, t1, device="cuda")[:, None] - torch.arange(t1, device="cuda")[None]
                w = torch.where(gap >= 0, power[gap.clamp(min=0)], 0.0)
                for h in range(j * group, (j + 1) * group):
                    row = st["q"][b, t0:t1, h].double()
                    if not back:
                        o[b, t0:t1, h] = scale * ((row @ k[:t1].T * w) @ v[:t1] + since[t0:t1] * (row @ s0))
                        continue
                    up = st["d_o"][b, t0:t1, h].double() * scale
                    dp = up @ v[:t1].T * w
                    o[b, t0:t1, h] = dp @ k[:t1] + since[t0:t1] * (up @ s0.T)
                    dk[b, :t1, j] += dp.T @ row
                    dv[b, :t1, j] += (row @ k[:t1].T * w).T @ up
                    if c["carry"]:
                        state[b, j] += (since[t0:t1] * row).T @ up
            if c["carry"] and back:
                ds = st["d_state_out"][b, j].double()
                dk[b, :n, j] += left * (v @ ds.T)
                dv[b, :n, j] += left * (k @ ds)
                state[b, j] += torch.exp(log * n) * ds
            elif c["carry"]:
                state[b, j] = torch.exp(log * n) * s0 + (left * k).T @ v
    return [o, dk, dv, state] if back else [o, state]
