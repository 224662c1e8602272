"""Tokens into the paged cache and back, through the C ABI against the fp64 oracle.

Tolerances: rotated queries and a bf16 cache hold one rounding to bf16 (2^-8 of a value) on top of fp32 arithmetic (products of two values, rounded each, and
their sum: 3 * 2^-24 of the pair's magnitude).  Of an e4m3 cache the exponents and codes of unrotated vectors are those of the oracle, bit for bit; of rotated
vectors, whose fp32 values may lie on the other side of a rounding's tie, one step of e4m3 (2^-3 of a value's binade, 2^-9 of the smallest) more than half a step.
"""
import numpy as np
import pytest
import torch

from oracle import generation as og
from synth import inputs as si
from tests.paged import Pages, bits, garbage, i64
from tests.parity import dev_bf16, host_f64

pytestmark = pytest.mark.gpu

BF16 = 2.0 ** -8 * 1.001


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


# tokens before, tokens of the call, seq, query heads, KV heads, head_dim, page
CASES = {
    "one": ([5], None, 1, 4, 2, 128, 16),
    "decode": ([0, 15, 16, 77, 500], None, 1, 8, 2, 128, 16),
    "idle_rows": ([3, 9, 30], [1, 0, 1], 1, 3, 1, 32, 32),
    "ragged": ([0, 33, 200, 5], [0, 37, 70, 1], 70, 6, 2, 64, 16),
    "odd_heads": ([7, 0], [50, 300], 300, 7, 5, 32, 64),
    "prompt": ([0, 0], None, 257, 4, 4, 128, 256),
}


def tokens(rng, case, std=1.3):
    start, lengths, s, hq, hkv, dh, _ = case
    b = len(start)
    return bits(rng, (b, s, hq, dh), std), bits(rng, (b, s, hkv, dh), std), bits(rng, (b, s, hkv, dh))


def spoiled(t, lengths):
    t = t.clone()
    for b, n in enumerate(lengths or []):
        t[b, n:] = float("nan")
    return t


def new_positions(case):
    start, lengths, s = case[:3]
    for b, (a, n) in enumerate(zip(start, lengths or [s] * len(start))):
        for t in range(n):
            yield b, t, a + t


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("name", list(CASES))
def test_append_without_rotation_and_read(K, name, e4m3):
    """What is held is the oracle's, bit for bit, everything else in the cache stays as it was, and reading gives what is held."""
    case = CASES[name]
    start, lengths, s, hq, hkv, dh, page = case
    rng = np.random.default_rng(len(name) + 17 * e4m3)
    n = lengths or [s] * len(start)
    pages = Pages(rng, [a + m for a, m in zip(start, n)], hkv, dh, page, e4m3)
    cache = pages.device(K)
    _, kb, vb = tokens(rng, case)
    K.kv_cache_append(cache, None, spoiled(dev_bf16(kb), lengths), spoiled(dev_bf16(vb), lengths), i64(start), i64(lengths), s, 0, 0.0, 0, None)
    for b, t, p in new_positions(case):
        pages.put(0, b, p, kb[b, t])
        pages.put(1, b, p, vb[b, t])
    want = pages.device(K)
    for got, ref in zip(cache.tensors, want.tensors):
        assert (got is None and ref is None) or torch.equal(got.view(torch.uint8), ref.view(torch.uint8))
    out = [garbage((len(start), s, hkv, dh)) for _ in range(2)]
    K.kv_cache_read(cache, i64(start), i64(lengths), s, *out)
    held = pages.oracle()
    ref = {w: np.zeros((len(start), s, hkv, dh)) for w in "kv"}
    for b, t, p in new_positions(case):
        pg, slot = og.place(held, b, p)
        for w in "kv":
            ref[w][b, t] = held[w][pg, :, slot]
    for got, w in zip(out, "kv"):
        assert np.array_equal(host_f64(got), ref[w])


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("name", list(CASES))
def test_append_with_rotation(K, name, e4m3, layout):
    case = CASES[name]
    start, lengths, s, hq, hkv, dh, page = case
    rng = np.random.default_rng(len(name) + 17 * e4m3 + 5 * layout)
    n = lengths or [s] * len(start)
    far = [a + 30000 if s == 1 else a for a in start]                      # a row's position is its place: far only where few pages are needed
    pages = Pages(rng, [0] * len(start), hkv, dh, page, e4m3, columns=max(-(-(a + m) // page) for a, m in zip(far, n)), spare=sum(m // page + 2 for m in n))
    free = list(range(pages.shape[0]))
    for b, (a, m) in enumerate(zip(far, n)):
        for c in range(a // page, -(-(a + m) // page)):
            pages.table[b, c] = free.pop()
    cache = pages.device(K)
    qb, kb, vb = tokens(rng, case)
    q_out = garbage(qb.shape)
    K.kv_cache_append(cache, spoiled(dev_bf16(qb), lengths), spoiled(dev_bf16(kb), lengths), spoiled(dev_bf16(vb), lengths), i64(far), i64(lengths), s, hq,
                      5e5, layout, q_out)
    got_q, ref_q = host_f64(q_out), np.zeros(qb.shape)
    codes = [t.cpu().view(torch.uint8).numpy() if e4m3 else host_f64(t) for t in cache.tensors[:2]]
    scales = [t.cpu().numpy().astype(np.int64) - 127 if e4m3 else None for t in cache.tensors[2:4]]
    written = np.zeros(pages.shape[:3], bool)
    for b, t, _ in new_positions(case):
        p = far[b] + t
        ref_q[b, t] = og.rotate(si.bf16_bits_to_f64(qb[b, t]), p, 5e5, layout)
        pg, slot = og.place({"k": np.empty(pages.shape), "page_table": pages.table}, b, p)
        written[pg, :, slot] = True
        k = og.rotate(si.bf16_bits_to_f64(kb[b, t]), p, 5e5, layout)
        v = si.bf16_bits_to_f64(vb[b, t])
        if e4m3:
            for w, x in ((0, k), (1, v)):
                held, e = og.dequantise(codes[w][pg, :, slot], scales[w][pg, :, slot]), og.quantise(x)[1]
                step = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 1e-30))) - 3), 2.0 ** (e[:, None] - 9.0))
                assert np.all(np.abs(held - x) <= step * (0.5 if w else 0.5001)) and np.array_equal(scales[w][pg, :, slot], e)
        else:
            assert np.array_equal(codes[1][pg, :, slot], v)
            assert np.all(np.abs(codes[0][pg, :, slot] - k) <= BF16 * np.abs(k) + 1e-6)
    assert np.all(np.abs(got_q - ref_q) <= BF16 * np.abs(ref_q) + 1e-6)
    for c in codes:                                                        # what no token was written to
        left = c[~written]
        assert np.all(left == 0xFF) if e4m3 else np.all(np.isnan(left))
    # in place, and the same bits
    q = spoiled(dev_bf16(qb), lengths)
    K.kv_cache_append(cache, q, dev_bf16(kb), dev_bf16(vb), i64(far), i64(lengths), s, hq, 5e5, layout, q)
    assert torch.equal(q.view(torch.int16), q_out.view(torch.int16))


def test_values_of_every_kind(K):
    """Zeros, the ends of the range, ties, and what is not finite, as one vector each; and every bf16 of a binade next to a large one."""
    dh = 128
    rows = [np.zeros(dh), np.full(dh, -0.0), np.full(dh, 3.3895313892515355e38), np.full(dh, 1e-38), np.linspace(-448, 448, dh), np.linspace(-449, 449, dh),
            np.where(np.arange(dh) == 3, np.inf, 1.0), np.where(np.arange(dh) == 3, -np.inf, 3.0), np.where(np.arange(dh) == 7, np.nan, 2.5), np.full(dh, np.nan),
            np.concatenate([[448.0], 2.0 ** -9 * np.arange(127) / 4]), np.concatenate([[1.0], 1 + np.arange(127) / 128]), np.full(dh, 1.75), np.full(dh, 1.7578125)]
    x = si.f32_to_bf16_bits(np.array(rows, np.float32))[None, :, None]                # [1, rows, 1, dh]
    n = len(rows)
    rng = np.random.default_rng(0)
    pages = Pages(rng, [n], 1, dh, 16, True)
    cache = pages.device(K)
    t = dev_bf16(x)
    K.kv_cache_append(cache, None, t, t.flip(1).contiguous(), None, None, n, 0, 0.0, 0, None)
    for p in range(n):
        pages.put(0, 0, p, x[0, p])
        pages.put(1, 0, p, x[0, n - 1 - p])
    want = pages.device(K)
    for got, ref in zip(cache.tensors[:2], want.tensors[:2]):
        nan = (ref & 127) == 127
        assert torch.equal((got & 127) == 127, nan)                                  # a NaN's sign is nobody's
        assert torch.equal(got[~nan], ref[~nan])
    for got, ref in zip(cache.tensors[2:], want.tensors[2:]):
        assert torch.equal(got, ref)
    out = [garbage((1, n, 1, dh)) for _ in range(2)]
    K.kv_cache_read(cache, None, None, n, *out)
    held = pages.oracle()["k"][pages.table[0, 0]][0][:n]
    assert np.array_equal(host_f64(out[0])[0, :, 0], held, equal_nan=True)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_places_that_do_not_exist(K, e4m3):
    """Nothing is written for them and nothing but zeros read; the tokens beside them are."""
    rng = np.random.default_rng(1)
    hkv, dh, s = 2, 64, 40
    pages = Pages(rng, [160, 160, 160, 160, 160], hkv, dh, 16, e4m3, columns=10)
    pages.table[0, 1] = -1
    pages.table[1, 2] = pages.shape[0]
    start = [0, 0, 140, -20, 1 << 62]
    cache = pages.device(K)
    kb, vb = bits(rng, (5, s, hkv, dh)), bits(rng, (5, s, hkv, dh))
    K.kv_cache_append(cache, None, dev_bf16(kb), dev_bf16(vb), i64(start), None, s, 0, 0.0, 0, None)
    out = [garbage((5, s, hkv, dh)) for _ in range(2)]
    K.kv_cache_read(cache, i64(start), None, s, *out)
    there = np.zeros((5, s), bool)
    for b, a in enumerate(start):
        for t in range(s):
            if og.place({"k": np.empty(pages.shape), "page_table": pages.table}, b, a + t) is not None:
                there[b, t] = True
                pages.put(0, b, a + t, kb[b, t])
                pages.put(1, b, a + t, vb[b, t])
    assert there.sum() == 24 + 32 + 20 + 20
    want = pages.device(K)
    for got, ref in zip(cache.tensors, want.tensors):
        assert (got is None and ref is None) or torch.equal(got.view(torch.uint8), ref.view(torch.uint8))
    held = pages.oracle()
    for got, w in zip(out, "kv"):
        got = host_f64(got)
        assert np.all(got[~there] == 0)
        for b, t in zip(*there.nonzero()):
            pg, slot = og.place(held, b, start[b] + t)
            assert np.array_equal(got[b, t], held[w][pg, :, slot])


def test_captured_and_replayed(K):
    """One step of generation as a graph: positions and tokens change between replays, eager work in between."""
    rng = np.random.default_rng(4)
    hq, hkv, dh = 4, 2, 64
    pages = Pages(rng, [100, 100], hkv, dh, 16, True)
    cache, mirror = pages.device(K), pages.device(K)
    q, k, v = (torch.empty((2, 1, h, dh), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    q_out, start = garbage(q.shape), torch.zeros(2, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        K.kv_cache_append(cache, q, k, v, start, None, 1, hq, 1e4, 0, q_out)
        start.add_(1)
    start.copy_(i64([3, 50]))
    for turn in range(4):
        for t in (q, k, v):
            t.copy_(dev_bf16(bits(rng, tuple(t.shape))))
        g.replay()
        torch.cuda.synchronize()
        eager = garbage(q.shape)
        K.kv_cache_append(mirror, q, k, v, i64([3 + turn, 50 + turn]), None, 1, hq, 1e4, 0, eager)
        assert torch.equal(q_out, eager)
        for a, b in zip(cache.tensors, mirror.tensors):
            assert torch.equal(a, b)


def test_a_cache_of_more_than_4_gib(K):
    hkv, dh, page = 8, 128, 64
    for dtype, size in ((torch.bfloat16, 2), (torch.uint8, 1)):
        n_pages = (5 << 30) // (hkv * page * dh * size)
        x = [torch.zeros((n_pages, hkv, page, dh), dtype=dtype, device="cuda") for _ in range(2)]
        s = [torch.full((n_pages, hkv, page), 127, dtype=torch.uint8, device="cuda") if size == 1 else None for _ in range(2)]
        ids = [n_pages - 1, 5, n_pages - 3]
        cache = K.KVCache.of(*x, torch.tensor([ids], dtype=torch.int32, device="cuda"), *s)
        k, v = (torch.randint(-8, 9, (1, 150, hkv, dh), device="cuda").bfloat16() for _ in range(2))    # exact in e4m3
        K.kv_cache_append(cache, None, k, v, None, None, 150, 0, 0.0, 0, None)
        out = [garbage(k.shape) for _ in range(2)]
        K.kv_cache_read(cache, None, None, 150, *out)
        assert torch.equal(out[0], k) and torch.equal(out[1], v)
        assert x[0][6:n_pages - 3].view(torch.uint8).max() == 0
        del x, s, cache


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_more_tokens_than_workgroups(K, e4m3):
    """A wave takes several tokens one after the other: the same bits as token by token."""
    b, s, hq, hkv, dh, page = 3, 3001, 3, 1, 32, 16
    columns = -(-s // page)
    table = torch.randperm(b * columns, device="cuda").view(b, columns).to(torch.int32)
    lengths = [s, 0, 1777]
    q, k, v = (torch.randn((b, s, h, dh), device="cuda").bfloat16() for h in (hq, hkv, hkv))
    caches, outs = [], []
    for _ in range(2):
        x = [torch.zeros((b * columns, hkv, page, dh), dtype=torch.uint8 if e4m3 else torch.bfloat16, device="cuda") for _ in range(2)]
        sc = [torch.zeros((b * columns, hkv, page), dtype=torch.uint8, device="cuda") if e4m3 else None for _ in range(2)]
        caches.append(K.KVCache.of(*x, table, *sc))
        outs.append(garbage(q.shape))
    K.kv_cache_append(caches[0], q, k, v, None, i64(lengths), s, hq, 1e4, 1, outs[0])
    for t0 in range(0, s, 500):
        n = min(500, s - t0)
        piece = [x[:, t0:t0 + n].contiguous() for x in (q, k, v)]
        out = garbage(piece[0].shape)
        K.kv_cache_append(caches[1], *piece, i64([t0] * b), i64([min(max(m - t0, 0), n) for m in lengths]), n, hq, 1e4, 1, out)
        outs[1][:, t0:t0 + n] = out
    assert torch.equal(outs[0], outs[1])
    for x, y in zip(caches[0].tensors, caches[1].tensors):
        assert (x is None and y is None) or torch.equal(x, y)
    got = [garbage(k.shape) for _ in range(2)]
    K.kv_cache_read(caches[0], None, i64(lengths), s, *got)
    assert all((x[1] == 0).all() and (x[2, 1777:] == 0).all() for x in got)
    if not e4m3:
        assert torch.equal(got[1][0], v[0]) and torch.equal(got[1][2, :1777], v[2, :1777])
