"""Generating with the softmax attention: a paged cache of keys and values, attention of new tokens over it, and log-probabilities of
tokens. The calls that these operators' performance is judged on, at the sizes their users run, with the operators' plain form in
elementary torch operations.

Kinds of cases
  append    kv_cache_append: new keys and values go to their pages (in bf16, or quantised to e4m3 with a power of two for each token and
            head); keys, and the queries beside them, are rotated to their positions on the way
  read      kv_cache_read: keys and values of consecutive tokens back from their pages, in bf16
  attend    paged_attention_forward: queries of seq new tokens a row, whose keys are in the cache already, over all keys up to their own
  logprobs  token_logprobs_forward ("forward") or token_logprobs_backward ("backward")

context: tokens in the cache before the new ones; contexts "ragged": row i of a batch has about (i + 1) / batch of them.
lengths: "full", or "ragged": row i of a batch holds about i / (batch - 1) of seq tokens (the first none, the last all), the rest is padding.
unscored: the share of rows without a token to score (padding of a batch of answers).
"""
import math

import torch

own = False

TOP = 448.0              # the largest value of e4m3


# ------------------------------------------------------------------ the cases
def _cached(kind, batch, seq, context, n_q_heads, n_kv_heads, head_dim, dtype, page, rope_layout=0, contexts="full", lengths="full", name=None):
    c = dict(kind=kind, batch=batch, seq=seq, context=context, n_q_heads=n_q_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, dtype=dtype,
             page=page, rope_layout=rope_layout, contexts=contexts, lengths=lengths)
    return dict(c, name=name) if name else c


def _logprobs(direction, rows, vocab, ld, n_top=0, temperature=1.0, unscored=0.0, name=None):
    c = dict(kind="logprobs", direction=direction, rows=rows, vocab=vocab, ld=ld, n_top=n_top, temperature=temperature, unscored=unscored)
    return dict(c, name=name) if name else c


def listed():
    return [
        # generating one sequence with an 8B-shaped model: one token's heads rotated and cached, nothing but latency
        _cached("append", 1, 1, 8000, 32, 8, 128, "e4m3", 16, name="append_1"),
        # two prompts of the 8B-shaped layer go to the cache
        _cached("append", 2, 8192, 0, 32, 8, 128, "e4m3", 64, name="append_prompt"),
        # the same prompts' keys and values back, for an operator that wants them in a row
        _cached("read", 2, 8192, 0, 32, 8, 128, "e4m3", 64, name="read_prompt"),
        # texts of different lengths, one of them empty, heads of 64, small pages
        _cached("read", 5, 1037, 211, 18, 6, 64, "bf16", 16, contexts="ragged", lengths="ragged", name="read_ragged"),
        # generating one sequence behind a long prompt
        _cached("attend", 1, 1, 32767, 32, 8, 128, "e4m3", 16, name="attend_1"),
        # generating many sequences of different lengths at once
        _cached("attend", 256, 1, 4095, 32, 8, 128, "bf16", 16, contexts="ragged", name="attend_256"),
        # pieces of prompts, of different lengths, behind what is cached of them already
        _cached("attend", 5, 1037, 8009, 32, 8, 128, "e4m3", 16, contexts="ragged", lengths="ragged", name="attend_chunk"),
        # two whole prompts at once
        _cached("attend", 2, 8192, 0, 32, 8, 128, "bf16", 64, name="attend_prompt"),
        # the token just generated, with the 20 likeliest in its place
        _logprobs("forward", 1, 128256, 128256, n_top=20, name="logprobs_1"),
        # scoring answers: every token's log-probability, the entropy and the 5 likeliest
        _logprobs("forward", 4096, 128256, 128256, n_top=5, name="logprobs_answers"),
        # the gradient of a policy's loss and its entropy bonus, the vocabulary padded for the product before it, part of the rows padding
        _logprobs("backward", 1037, 50257, 50304, temperature=0.7, unscored=0.2, name="logprobs_padded_grad"),
        _logprobs("backward", 4096, 128256, 128256, name="logprobs_answers_grad"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    largest = max(_cost(c) for c in listed())
    while True:
        if rng.random() < 0.3:
            direction = rng.choice(("forward", "forward", "backward"))
            vocab = _log_int(rng, 1000, 160000)
            c = _logprobs(direction, _log_int(rng, 1, 8192), vocab, -(-vocab // 8) * 8 + rng.choice((0, 0, 56)),
                          rng.choice((0, 1, 5, 20, 33, 64)) if direction == "forward" else 0, rng.choice((1.0, 1.0, 0.7, 1.3)), rng.choice((0.0, 0.0, 0.3)))
            if _cost(c) <= largest and c["rows"] * c["ld"] <= 1 << 30:
                return c
            continue
        head_dim = rng.choice((32, 64, 64, 128, 128, 128))
        n_kv_heads = _log_int(rng, 1, 16)
        n_q_heads = n_kv_heads * rng.choice((1, 1, 2, 3, 4, 8))
        if n_q_heads * head_dim > 4096:
            continue
        kind = rng.choice(("append", "append", "read", "attend", "attend", "attend", "attend"))
        seq = rng.choice((1, 1, rng.randint(2, 8), _log_int(rng, 9, 8192), _log_int(rng, 9, 8192)))
        batch = _log_int(rng, 1, 512) if seq <= 8 else rng.randint(1, 8)
        context = rng.choice((0, _log_int(rng, 1, 65536), _log_int(rng, 1, 65536)))
        c = _cached(kind, batch, seq, context, n_q_heads, n_kv_heads, head_dim, rng.choice(("bf16", "e4m3")), rng.choice((16, 16, 32, 64, 128, 256)),
                    rng.choice((0, 0, 1)), rng.choice(("full", "ragged")), rng.choice(("full", "full", "ragged")))
        if c["lengths"] == "ragged" and batch == 1:
            continue
        tokens, worst = batch * (context + seq), max(_scores(x) for x in listed())
        if tokens * n_kv_heads * head_dim <= 1 << 31 and _scores(c) <= worst and _cost(c) <= largest:
            return c


def _scores(c):
    """Elements of the scores that the plain form holds at once."""
    return c["batch"] * c["n_q_heads"] * c["seq"] * (c["context"] + c["seq"]) if c["kind"] == "attend" else 0


def _cost(c):
    """Bytes and operations on one scale, of the padded sizes: what a drawn case is held to."""
    w = work(dict(c, unscored=0.0) if c["kind"] == "logprobs" else dict(c, lengths="full", contexts="full"))
    return w["bytes"] + w["flops"] / 50


# ------------------------------------------------------------------ inputs
def _rows(c):
    """(tokens cached before the call, new tokens) of each batch row, from the case alone."""
    b, ctx, s = c["batch"], c["context"], c["seq"]
    starts = [ctx] * b if c["contexts"] == "full" else [ctx * (i + 1) // b for i in range(b)]
    return starts, [s] * b if c["lengths"] == "full" else [s * i // (b - 1) for i in range(b)]


def _scored(c):
    return c["rows"] - int(c["rows"] * c["unscored"])


def _quantised(x):
    """(e4m3 values, exponents with a bias of 127 as bytes) of vectors along the last axis: the smallest power of two that brings the vector within e4m3."""
    m, e = torch.frexp(x.float().abs().amax(-1) / TOP)            # amax / TOP = m 2^e, 0.5 <= m < 1
    e = torch.where(m == 0.5, e - 1, e).clamp(-126, 127)          # zeros get exponent 0
    return torch.ldexp(x.float(), -e[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen).to(dtype)

    st = {"case": c}
    if c["kind"] == "logprobs":
        # a model's logits: a normal spread of 2.5, of which the rows' likeliest tokens hold most of the probability; what lies behind the vocabulary is anything
        st["logits"] = normal(c["rows"], c["ld"], std=2.5)
        p = torch.softmax(st["logits"][:, :c["vocab"]].float() / c["temperature"], -1)
        st["targets"] = torch.multinomial(p, 1, generator=gen)[:, 0]
        st["targets"][_scored(c):] = -1
        if c["direction"] == "backward":
            st["d_logprobs"] = normal(c["rows"], dtype=torch.float32)                       # advantages
            st["d_entropy"] = torch.full((c["rows"],), 0.01, device="cuda")
            st["lse"], st["entropy"] = _plain_statistics(st, c)[2:]                         # what the forward left
        return st
    b, s, hq, hkv, dh, page = c["batch"], c["seq"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"], c["page"]
    starts, lengths = _rows(c)
    st["start"] = torch.tensor(starts, dtype=torch.int64, device="cuda")
    st["lengths"] = None if c["lengths"] == "full" else torch.tensor(lengths, dtype=torch.int64, device="cuda")
    # pages in the order in which a long-running program's free list gives them out, -1 where a row has none
    columns = max(1, -(-(c["context"] + s) // page))
    held = torch.tensor([-(-(n + m) // page) for n, m in zip(starts, lengths)], device="cuda")
    table = torch.randperm(b * columns, generator=gen, device="cuda").view(b, columns)
    st["page_table"] = torch.where(torch.arange(columns, device="cuda") < held[:, None], table, -1).to(torch.int32)
    # queries and keys whose scores spread as a trained model's do; values of a deviation of one
    for name in ("k", "v"):
        x = normal(b * columns, hkv, page, dh, std=1.0)
        st[name + "_cache"], st[name + "_scale"] = _quantised(x) if c["dtype"] == "e4m3" else (x, None)
    if c["kind"] != "read":
        st["q"] = normal(b, s, hq, dh, std=1.3)
    if c["kind"] == "append":
        st["k"], st["v"] = normal(b, s, hkv, dh, std=1.3), normal(b, s, hkv, dh)
    return st


# ------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if own:
        return _own_logprobs(state, c) if c["kind"] == "logprobs" else _own_cached(state, c)
    if c["kind"] == "logprobs":
        return _plain_logprobs_backward(state, c) if c["direction"] == "backward" else _plain_logprobs(state, c)
    return {"append": _plain_append, "read": _plain_read, "attend": _plain_attend}[c["kind"]](state, c)


ROPE_BASE = 5e5


def _own_cached(st, c):
    import paper_2602_08387_amd as K
    if "cache" not in st:          # a program's handle, its output buffers and its workspace, kept from step to step
        st["cache"] = K.KVCache.of(st["k_cache"], st["v_cache"], st["page_table"], st["k_scale"], st["v_scale"])
        if c["kind"] == "read":
            st["out"] = [torch.empty((c["batch"], c["seq"], c["n_kv_heads"], c["head_dim"]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        else:
            st["out"] = [torch.empty_like(st["q"])]
        if c["kind"] == "attend":
            st["out"].append(torch.empty((c["batch"], c["n_q_heads"], c["seq"]), dtype=torch.float32, device="cuda"))
            st["ws"] = torch.empty(K.paged_attention_workspace_bytes(st["cache"], c["seq"], c["n_q_heads"]), dtype=torch.uint8, device="cuda")
    if c["kind"] == "append":
        K.kv_cache_append(st["cache"], st["q"], st["k"], st["v"], st["start"], st["lengths"], c["seq"], c["n_q_heads"], ROPE_BASE, c["rope_layout"],
                          st["out"][0])
        return st["out"] + [st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"]]
    if c["kind"] == "read":
        K.kv_cache_read(st["cache"], st["start"], st["lengths"], c["seq"], *st["out"])
    else:
        K.paged_attention_forward(st["cache"], st["q"], st["start"], st["lengths"], c["seq"], c["n_q_heads"], c["head_dim"] ** -0.5, *st["out"], st["ws"])
    return st["out"]


def _own_logprobs(st, c):
    import paper_2602_08387_amd as K
    rows, vocab, ld, n_top, inverse = c["rows"], c["vocab"], c["ld"], c["n_top"], 1.0 / c["temperature"]
    if c["direction"] == "backward":
        if "out" not in st:
            st["out"] = [torch.empty_like(st["logits"])]
        K.token_logprobs_backward(st["logits"], st["targets"], st["lse"], st["entropy"], st["d_logprobs"], st["d_entropy"], rows, vocab, ld, inverse,
                                  st["out"][0])
        return st["out"]
    if "out" not in st:
        st["out"] = [torch.empty(rows, dtype=torch.float32, device="cuda") for _ in range(3)]
        st["out"] += [torch.empty((rows, n_top), dtype=t, device="cuda") if n_top else None for t in (torch.int64, torch.float32)]
        st["ws"] = torch.empty(K.token_logprobs_workspace_bytes(rows, vocab, n_top), dtype=torch.uint8, device="cuda")
    K.token_logprobs_forward(st["logits"], st["targets"], rows, vocab, ld, inverse, n_top, *st["out"], st["ws"])
    return st["out"]


# ------------------------------------------------------------------ the plain form: the cache
def _positions(st, c):
    """Positions [batch, seq] of the new tokens, and whether each is one (and not padding)."""
    t = torch.arange(c["seq"], device="cuda")
    n = st["lengths"]
    valid = torch.ones((c["batch"], c["seq"]), dtype=torch.bool, device="cuda") if n is None else t < n[:, None]
    return st["start"][:, None] + t, valid


def _places(st, c):
    """(batch row, token, page, slot) of every new token that is one."""
    p, valid = _positions(st, c)
    row, t = valid.nonzero(as_tuple=True)
    p = p[row, t]
    return row, t, st["page_table"][row, p // c["page"]].long(), p % c["page"]


def _values(cache, scale):
    """What the cache holds, in 32 bits."""
    return cache.float() if scale is None else torch.ldexp(cache.float(), scale.int()[..., None] - 127)


def _halves(x, layout):
    return (x[..., 0::2], x[..., 1::2]) if layout else x.chunk(2, -1)


def _joined(a, b, layout):
    return torch.stack((a, b), -1).flatten(-2) if layout else torch.cat((a, b), -1)


def _plain_append(st, c):
    p, valid = _positions(st, c)
    theta = ROPE_BASE ** (-2.0 * torch.arange(c["head_dim"] // 2, dtype=torch.float64, device="cuda") / c["head_dim"])
    phi = p.double()[..., None, None] * theta
    cos, sin = phi.cos().float(), phi.sin().float()

    def rotated(x):
        a, b = _halves(x.float(), c["rope_layout"])
        return _joined(a * cos - b * sin, b * cos + a * sin, c["rope_layout"])

    q_out = torch.where(valid[..., None, None], rotated(st["q"]), 0.0).bfloat16()
    row, t, page, slot = _places(st, c)
    for name, x in (("k", rotated(st["k"])), ("v", st["v"].float())):
        x = x[row, t]                                              # [tokens, heads, head_dim]
        if c["dtype"] == "e4m3":
            x, scale = _quantised(x)
            st[name + "_cache"].view(torch.uint8)[page, :, slot] = x.view(torch.uint8)
            st[name + "_scale"][page, :, slot] = scale
        else:
            st[name + "_cache"][page, :, slot] = x.bfloat16()
    return [q_out, st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"]]


def _plain_read(st, c):
    row, t, page, slot = _places(st, c)
    out = [torch.zeros((c["batch"], c["seq"], c["n_kv_heads"], c["head_dim"]), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for o, name in zip(out, ("k", "v")):
        scale = st[name + "_scale"]
        x = st[name + "_cache"].view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn) if c["dtype"] == "e4m3" else st[name + "_cache"][page, :, slot]
        o[row, t] = _values(x, None if scale is None else scale[page, :, slot]).bfloat16()
    return out


# ------------------------------------------------------------------ the plain form: attention
def _plain_attend(st, c):
    b, s, hq, hkv, dh = c["batch"], c["seq"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    p, valid = _positions(st, c)
    p = torch.where(valid, p, -1)
    table = st["page_table"].clamp(min=0).long()
    n = table.shape[1] * c["page"]
    ends = p.amax(-1) + 1                                          # keys of each row
    kept = (torch.arange(n, device="cuda") < ends[:, None])[:, None, :, None]

    def in_a_row(name):
        """[batch, kv head, token, head_dim] in 32 bits, zeros behind the last key."""
        pages = st[name + "_cache"].view(torch.uint8)[table].view(st[name + "_cache"].dtype)
        scale = st[name + "_scale"]
        x = _values(pages, None if scale is None else scale[table])
        return x.transpose(1, 2).reshape(b, hkv, n, dh).masked_fill_(~kept, 0.0)

    k, v = in_a_row("k"), in_a_row("v")
    q = st["q"].float().view(b, s, hkv, -1, dh).permute(0, 2, 3, 1, 4)          # [batch, kv head, head of its group, token, head_dim]
    g = q.shape[2]
    x = (q.reshape(b, hkv, g * s, dh) @ k.transpose(-1, -2)).mul_(dh ** -0.5).view(b, hkv, g, s, n)
    x.masked_fill_((torch.arange(n, device="cuda") > p[..., None])[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top.clamp(min=-1e30)).exp_()
    total = x.sum(-1, keepdim=True)
    o = (x.view(b, hkv, g * s, n) @ v).view(b, hkv, g, s, dh) / total.clamp(min=1e-30)
    lse = (top + total.log())[..., 0]
    return [o.permute(0, 3, 1, 2, 4).reshape(b, s, hq, dh).bfloat16(), lse.reshape(b, hq, s)]


# ------------------------------------------------------------------ the plain form: log-probabilities
def _plain_statistics(st, c):
    """(log-probabilities [rows, vocab], whether a row counts, log-sum-exp and entropy of each row or 0)."""
    z = st["logits"][:, :c["vocab"]].float() * (1.0 / c["temperature"])
    counts = (st["targets"] >= 0) & (st["targets"] < c["vocab"])
    top = z.amax(-1, keepdim=True)
    t = z - top
    e = t.exp()
    total = e.sum(-1, keepdim=True)
    entropy = (total.log() - (e * t).sum(-1, keepdim=True) / total)[:, 0]
    lse = top + total.log()
    return z - lse, counts, torch.where(counts, lse[:, 0], 0.0), torch.where(counts, entropy, 0.0)


def _plain_logprobs(st, c):
    logp, counts, lse, entropy = _plain_statistics(st, c)
    chosen = torch.where(counts, logp.gather(1, st["targets"].clamp(min=0)[:, None])[:, 0], 0.0)
    if not c["n_top"]:
        return [chosen, entropy, lse, None, None]
    # an order without ties: the logit's bits as a whole number of the same order, then the lower index
    bits = st["logits"][:, :c["vocab"]].contiguous().view(torch.int16).long()
    order = torch.where(bits >= 0, bits, -32768 - bits)
    ids = ((order << 32) - torch.arange(c["vocab"], device="cuda")).topk(c["n_top"], dim=-1).indices
    return [chosen, entropy, lse, torch.where(counts[:, None], ids, -1), torch.where(counts[:, None], logp.gather(1, ids), 0.0)]


def _plain_logprobs_backward(st, c):
    inverse = 1.0 / c["temperature"]
    counts = ((st["targets"] >= 0) & (st["targets"] < c["vocab"]))[:, None]
    logp = st["logits"][:, :c["vocab"]].float() * inverse - st["lse"][:, None]
    d = -logp.exp() * (st["d_logprobs"][:, None] + st["d_entropy"][:, None] * (logp + st["entropy"][:, None]))
    d.scatter_add_(1, st["targets"].clamp(min=0)[:, None], st["d_logprobs"][:, None])
    d = torch.where(counts, d * inverse, 0.0)
    return [torch.nn.functional.pad(d, (0, c["ld"] - c["vocab"])).bfloat16()]


# ------------------------------------------------------------------ what cannot be done without
def work(case):
    c = case
    if c["kind"] == "logprobs":
        n, row = _scored(c), c["vocab"]
        if c["direction"] == "backward":
            return {"bytes": 2 * row * n + 2 * c["ld"] * c["rows"] + 24 * c["rows"], "flops": 8 * row * n}
        return {"bytes": 2 * row * n + (20 + 12 * c["n_top"]) * c["rows"], "flops": 7 * row * n}
    hq, hkv, dh = c["n_q_heads"], c["n_kv_heads"], c["head_dim"]
    starts, lengths = _rows(c)
    padded, tokens = c["batch"] * c["seq"], sum(lengths)
    held = 2 * hkv * (2 * dh if c["dtype"] == "bf16" else dh + 1)               # bytes of a token's keys and values in the cache
    if c["kind"] == "append":
        return {"bytes": tokens * (2 * (hq + 2 * hkv) * dh + held) + 2 * padded * hq * dh, "flops": (3 * hq + 7 * hkv) * dh * tokens}
    if c["kind"] == "read":
        return {"bytes": tokens * held + 4 * padded * hkv * dh, "flops": 2 * hkv * dh * tokens}
    seen = sum(n * a + n * (n + 1) // 2 for a, n in zip(starts, lengths))       # keys that the new tokens see
    keys = sum(a + n for a, n in zip(starts, lengths) if n)
    return {"bytes": keys * held + 2 * hq * dh * (tokens + padded) + 4 * hq * padded, "flops": 4 * hq * dh * seen}


# ------------------------------------------------------------------ the definitions in 64 bits
def _decoded(codes, scale):
    """e4m3 from its bits, times its power of two."""
    b = codes.view(torch.uint8).to(torch.int64)
    exponent, mantissa = (b >> 3) & 15, (b & 7).double()
    x = torch.where(exponent == 0, mantissa / 8 * 2.0 ** -6, (1 + mantissa / 8) * torch.exp2(exponent.double() - 7)) * (1 - 2 * (b >> 7)).double()
    return x if scale is None else x * torch.exp2(scale.double() - 127)[..., None]


def exact(case, seed):
    c, st = case, prepare(case, seed)
    f64 = dict(dtype=torch.float64, device="cuda")
    if c["kind"] == "logprobs":
        return _exact_backward(st, c) if c["direction"] == "backward" else _exact_logprobs(st, c)
    b, s, hq, hkv, dh, page = c["batch"], c["seq"], c["n_q_heads"], c["n_kv_heads"], c["head_dim"], c["page"]
    starts, lengths = _rows(c)

    def keys(name, row, first, end):
        """[token, kv head, head_dim] of one batch row."""
        ids = st["page_table"][row, first // page:-(-end // page)].long()
        x, scale = st[name + "_cache"], st[name + "_scale"]
        x = x[ids].double() if scale is None else _decoded(x.view(torch.uint8)[ids], scale[ids])
        return x.transpose(1, 2).reshape(-1, hkv, dh)[first % page:first % page + end - first]

    if c["kind"] == "read":
        out = [torch.zeros((b, s, hkv, dh), **f64) for _ in range(2)]
        for i, (a, n) in enumerate(zip(starts, lengths)):
            for o, name in zip(out, ("k", "v")):
                o[i, :n] = keys(name, i, a, a + n)
        return out

    if c["kind"] == "append":
        def turned(x, positions):
            theta = ROPE_BASE ** (-2.0 * torch.arange(dh // 2, **f64) / dh)
            turn = torch.polar(torch.ones((), **f64), positions[:, None, None] * theta)
            z = x.double().unflatten(-1, (-1, 2)) if c["rope_layout"] else x.double().unflatten(-1, (2, -1)).transpose(-1, -2)
            y = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            return (y if c["rope_layout"] else y.transpose(-1, -2)).flatten(-2)

        def held(x):
            """In units of its power of two, on the grid of e4m3."""
            e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / TOP))
            y = x / torch.exp2(e)
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -20))).clamp(min=-6) - 3)
            return torch.round(y / step) * step

        q_out = torch.zeros((b, s, hq, dh), **f64)
        out = [_decoded(st[n], None) if c["dtype"] == "e4m3" else st[n].double() for n in ("k_cache", "v_cache")]
        for i, (a, n) in enumerate(zip(starts, lengths)):
            p = torch.arange(a, a + n, **f64)
            q_out[i, :n] = turned(st["q"][i, :n], p)
            at = st["page_table"][i].long()[torch.arange(a, a + n, device="cuda") // page], torch.arange(a, a + n, device="cuda") % page
            for o, x in zip(out, (turned(st["k"][i, :n], p), st["v"][i, :n].double())):
                o[at[0], :, at[1]] = held(x) if c["dtype"] == "e4m3" else x
        return [q_out] + out + [None, None]

    # attention: one batch row and KV head after the other, some 2^26 scores at a time
    o, lse = torch.zeros((b, s, hq, dh), **f64), torch.full((b, hq, s), -math.inf, **f64)
    g = hq // hkv
    for i, (a, n) in enumerate(zip(starts, lengths)):
        if not n:
            continue
        k, v = keys("k", i, 0, a + n), keys("v", i, 0, a + n)
        some = max(1, (1 << 26) // (g * (a + n)))
        for j in range(hkv):
            for t0 in range(0, n, some):
                t1 = min(n, t0 + some)
                x = st["q"][i, t0:t1, j * g:(j + 1) * g].double().transpose(0, 1) @ k[:a + t1, j].T * dh ** -0.5
                x = torch.where(torch.arange(a + t1, device="cuda") <= torch.arange(a + t0, a + t1, device="cuda")[:, None], x, -math.inf)
                total = torch.logsumexp(x, -1)
                o[i, t0:t1, j * g:(j + 1) * g] = (torch.exp(x - total[..., None]) @ v[:a + t1, j]).transpose(0, 1)
                lse[i, j * g:(j + 1) * g, t0:t1] = total
    return [o, lse]


def _exact_logprobs(st, c):
    n = c["n_top"]
    out = [[], [], [], []]
    for x, tgt in zip(st["logits"].split(256), st["targets"].split(256)):
        z = x[:, :c["vocab"]].double() / c["temperature"]
        logp, counts = torch.log_softmax(z, -1), tgt >= 0
        rows = (logp.gather(1, tgt.clamp(min=0)[:, None])[:, 0], -(logp.exp() * logp).sum(-1), torch.logsumexp(z, -1), logp.topk(n, -1).values if n else None)
        for o, r in zip(out, rows):
            o.append(None if r is None else torch.where(counts if r.dim() == 1 else counts[:, None], r, 0.0))
    return [torch.cat(o) for o in out[:3]] + [None, torch.cat(out[3]) if n else None]


def _exact_backward(st, c):
    """By torch's differentiation of the definition."""
    out = torch.zeros(st["logits"].shape, dtype=torch.float64, device="cuda")
    for r in range(0, _scored(c), 128):
        at = slice(r, min(r + 128, _scored(c)))
        z = st["logits"][at, :c["vocab"]].double().requires_grad_()
        logp = torch.log_softmax(z / c["temperature"], -1)
        loss = (logp.gather(1, st["targets"][at, None])[:, 0] * st["d_logprobs"][at].double()).sum()
        loss = loss + (-(logp.exp() * logp).sum(-1) * st["d_entropy"][at].double()).sum()
        out[at, :c["vocab"]] = torch.autograd.grad(loss, z)[0]
    return [out]
