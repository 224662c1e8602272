"""Attention of new tokens over a paged cache, through the C ABI against the fp64 oracle.

Tolerances, from the arithmetic, element by element.  The operands (bf16, and e4m3 times a power of two) are exact in bf16, their products in fp32.
  scores    an fp32 sum of dh products is off by at most dh * 2^-24 of the sum of their magnitudes, `big` in the units of the exponent; the exponent and the
            exponential add a few units of 2^-24 of it: e = (dh + 8) * 2^-24 * (big + 1) for the relative error of a weight, and for the lse, which
            also is rounded itself
  result    each weight is rounded to bf16 for its product (2^-8), the result is rounded to bf16 (2^-8 of it): with mag = sum of weight * |v|,
            |error| <= (2^-8 + 2 e) * mag + 2^-8 * |o|, and 1 % for second orders and fp32 sums
"""
import numpy as np
import pytest
import torch

from oracle import generation as og
from synth import inputs as si
from tests.paged import Pages, bits, garbage, i64, workspace
from tests.parity import dev_bf16, host_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def spoiled(q, lengths):
    q = q.clone()
    for b, n in enumerate(lengths or []):
        q[b, max(0, n):] = float("nan")
    return q


def run(K, cache, q, start, lengths, n_q_heads, scale, with_lse=True, stream=None):
    b, s = q.shape[:2]
    o = garbage(q.shape)
    lse = garbage((b, n_q_heads, s), torch.float32) if with_lse else None
    ws = workspace(K.paged_attention_workspace_bytes(cache, s, n_q_heads))
    K.paged_attention_forward(cache, q, i64(start), i64(lengths), s, n_q_heads, scale, o, lse, ws, stream)
    return o, lse


def check(o, lse, ref, scale_dh):
    ref_o, ref_lse, mag, big = ref
    e = (scale_dh + 8) * 2.0 ** -24 * (big + 1)
    got_o, got_lse = host_f64(o), host_f64(lse)
    et = np.transpose(e, (0, 2, 1))[..., None]
    bound = 1.01 * ((2.0 ** -8 + 2 * et) * mag + 2.0 ** -8 * np.abs(ref_o)) + 1e-30
    worst = np.max(np.abs(got_o - ref_o) / bound)
    assert worst <= 1, worst
    empty = np.isneginf(ref_lse)
    assert np.array_equal(empty, np.isneginf(got_lse))
    off = np.abs(got_lse[~empty] - ref_lse[~empty]) / (2 * e[~empty] + 2.0 ** -22 * (np.abs(ref_lse[~empty]) + 1))
    assert off.size == 0 or off.max() <= 1, off.max()


# batch rows' tokens before the call, tokens of the call, seq, query and KV heads, head_dim, page
CASES = {
    "decode": ([0, 15, 16, 77, 300], None, 1, 8, 2, 128, 16),
    "decode_one_head": ([63, 64, 129], None, 1, 1, 1, 64, 32),
    "decode_some_idle": ([40, 7, 100], [1, 0, 1], 1, 16, 1, 32, 16),
    "decode_group_of_3": ([200, 31], None, 1, 9, 3, 64, 64),
    "decode_long": ([4000, 2111], None, 1, 8, 2, 128, 16),
    "few_tokens": ([0, 129, 30], [4, 4, 3], 4, 8, 2, 128, 16),
    "few_tokens_no_sharing": ([0, 65], None, 5, 3, 3, 32, 16),
    "16_rows": ([17, 0, 250], [8, 1, 7], 8, 4, 2, 64, 16),
    "17_rows": ([17, 0, 250], [17, 1, 16], 17, 2, 2, 64, 16),
    "whole_rows": ([0], None, 128, 4, 1, 128, 128),
    "ragged": ([0, 33, 200, 5], [0, 37, 70, 1], 70, 6, 2, 64, 16),
    "ragged_128": ([0, 33, 517], [129, 0, 61], 130, 8, 2, 128, 16),
    "ragged_32": ([3, 100], [65, 200], 201, 4, 4, 32, 256),
    "large_group": ([5, 90], None, 9, 64, 2, 32, 16),
}


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("name", list(CASES))
def test_against_the_oracle(K, name, e4m3):
    start, lengths, s, hq, hkv, dh, page = CASES[name]
    rng = np.random.default_rng(len(name) + e4m3)
    n = lengths or [s] * len(start)
    pages = Pages(rng, [a + m for a, m in zip(start, n)], hkv, dh, page, e4m3)
    qb = bits(rng, (len(start), s, hq, dh), 2.0)
    scale = dh ** -0.5
    cache = pages.device(K)
    o, lse = run(K, cache, spoiled(dev_bf16(qb), lengths), start, lengths, hq, scale)
    check(o, lse, og.attention(pages.oracle(), si.bf16_bits_to_f64(qb), start, lengths, scale), dh)
    # without the statistics, and into another result: the same bits
    again, _ = run(K, cache, spoiled(dev_bf16(qb), lengths), start, lengths, hq, scale, with_lse=False)
    assert torch.equal(o.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("s", [1, 6, 70])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_large_scores_and_means(K, s, e4m3):
    """Scores of some hundreds, keys and values with means: the running maximum is raised over and over."""
    rng = np.random.default_rng(s)
    start, hq, hkv, dh = [300, 81], 4, 2, 64
    pages = Pages(rng, [a + s for a in start], hkv, dh, 16, e4m3, std=4.0, mean=3.0)
    qb = bits(rng, (2, s, hq, dh), 4.0, 1.0)
    o, lse = run(K, pages.device(K), dev_bf16(qb), start, None, hq, 0.125)
    check(o, lse, og.attention(pages.oracle(), si.bf16_bits_to_f64(qb), start, None, 0.125), dh)


@pytest.mark.parametrize("s", [1, 5, 40])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_pages_that_do_not_exist(K, s, e4m3):
    """A page in the middle of a row, all pages of a row, and positions behind the table or before 0: not there."""
    rng = np.random.default_rng(7 + s)
    start, hq, hkv, dh = [120, 90, 200, -3, 1 << 40, -(1 << 63)], 4, 2, 64
    pages = Pages(rng, [120 + s, 90 + s, 160, s, 160, 160], hkv, dh, 16, e4m3, columns=10)
    pages.table[0, 3], pages.table[0, 4] = -5, 1 << 30
    pages.table[1] = -1
    qb = bits(rng, (6, s, hq, dh), 2.0)
    o, lse = run(K, pages.device(K), dev_bf16(qb), start, None, hq, 0.125)
    ref_start = [120, 90, 200, -3, 1000, -1000]
    ref = og.attention(pages.oracle(), si.bf16_bits_to_f64(qb), ref_start, None, 0.125)
    check(o, lse, ref, dh)


@pytest.mark.parametrize("s", [1, 33])
def test_rows_that_share_pages(K, s):
    rng = np.random.default_rng(3)
    pages = Pages(rng, [64 + s, 64 + s], 2, 128, 16, False)
    pages.table[1, :4] = pages.table[0, :4]
    qb = bits(rng, (2, s, 4, 128), 2.0)
    o, lse = run(K, pages.device(K), dev_bf16(qb), [64, 64], None, 4, 0.09)
    check(o, lse, og.attention(pages.oracle(), si.bf16_bits_to_f64(qb), [64, 64], None, 0.09), 128)


@pytest.mark.parametrize("s,group", [(3, 1), (3, 4), (40, 1), (70, 4)])
@pytest.mark.parametrize("what", ["v_inf", "v_nan", "k_nan"])
def test_values_that_are_not_finite_show_only_where_they_are_seen(K, s, group, what):
    rng = np.random.default_rng(s)
    at, hkv, dh, start = s - 1, 2, 64, 21
    pages = Pages(rng, [start + s], hkv, dh, 16, False)
    qb = bits(rng, (1, s, group * hkv, dh), 2.0)
    clean, clean_lse = run(K, pages.device(K), dev_bf16(qb), [start], None, group * hkv, 0.125)
    p = start + at
    bad = pages.codes[0 if what == "k_nan" else 1][pages.table[0, p // 16], 1, p % 16]
    bad[5] = 0x7F80 if what == "v_inf" else 0x7FC0
    o, lse = run(K, pages.device(K), dev_bf16(qb), [start], None, group * hkv, 0.125)
    o, clean = o.float(), clean.float()
    assert torch.equal(o[:, :at], clean[:, :at]) and torch.equal(o[:, :, :group], clean[:, :, :group])
    seen = o[0, at, group:]
    if what == "k_nan":
        assert seen.isnan().all() and lse[0, group:, at].isnan().all()
    else:
        assert not seen[:, 5].isfinite().any()
        rest = [d for d in range(dh) if d != 5]
        assert torch.equal(seen[:, rest], clean[0, at, group:][:, rest]) and torch.equal(lse, clean_lse)


def test_largest_magnitudes_of_the_quantised_cache(K):
    """Vectors near the ends of bf16's range, and zeros."""
    rng = np.random.default_rng(2)
    pages = Pages(rng, [40], 1, 32, 16, True)
    for p, scale in enumerate((3e38, 1e30, 1e-30, 1e-38, 0.0)):
        pages.put(1, 0, p, si.f32_to_bf16_bits((rng.uniform(-1, 1, (1, 32)) * scale).astype(np.float32)))
    qb = bits(rng, (1, 1, 2, 32), 1.0)
    o, lse = run(K, pages.device(K), dev_bf16(qb), [39], None, 2, 0.2)
    check(o, lse, og.attention(pages.oracle(), si.bf16_bits_to_f64(qb), [39], None, 0.2), 32)


@pytest.mark.parametrize("s", [1, 20])
def test_streams_and_graphs(K, s):
    """Captured once and replayed with other positions and other new tokens, with eager calls between; two graphs that share a workspace."""
    rng = np.random.default_rng(11)
    hq, hkv, dh = 4, 2, 64
    pages = Pages(rng, [300, 300], hkv, dh, 16, True)
    cache, oracle = pages.device(K), pages.oracle()
    q, start = torch.empty((2, s, hq, dh), dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    ws = workspace(K.paged_attention_workspace_bytes(cache, s, hq))
    outs = [(garbage(q.shape), garbage((2, hq, s), torch.float32)) for _ in range(2)]
    side, graphs = torch.cuda.Stream(), []
    torch.cuda.synchronize()
    for o, lse in outs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            K.paged_attention_forward(cache, q, start, None, s, hq, 0.125, o, lse, ws)
        graphs.append(g)
    for turn in range(4):
        qb, a = bits(rng, tuple(q.shape), 2.0), [int(x) for x in rng.integers(0, 300 - s, 2)]
        q.copy_(dev_bf16(qb))
        start.copy_(i64(a))
        for g, (o, lse) in zip(graphs, outs):
            o.fill_(float("nan"))
            g.replay()
        torch.cuda.synchronize()
        eager, eager_lse = run(K, cache, q, a, None, hq, 0.125)
        ref = og.attention(oracle, si.bf16_bits_to_f64(qb), a, None, 0.125)
        for o, lse in outs:
            check(o, lse, ref, dh)
            assert torch.equal(o.view(torch.int16), eager.view(torch.int16)) and torch.equal(lse, eager_lse)
    # on a stream that is not torch's current one
    o, lse = garbage(q.shape), garbage((2, hq, s), torch.float32)
    torch.cuda.synchronize()
    K.paged_attention_forward(cache, q, start, None, s, hq, 0.125, o, lse, ws, side)
    side.synchronize()
    assert torch.equal(o.view(torch.int16), outs[0][0].view(torch.int16))


@pytest.mark.parametrize("s", [1, 16, 200])
def test_nothing_is_written_around_the_outputs_and_the_workspace(K, s):
    rng = np.random.default_rng(5)
    hq, hkv, dh, guard = 4, 2, 128, 4096
    pages = Pages(rng, [700, 150], hkv, dh, 16, False, columns=60)
    cache = pages.device(K)
    before = [t.clone() for t in cache.tensors if t is not None]
    q = dev_bf16(bits(rng, (2, s, hq, dh), 2.0))
    nbytes = K.paged_attention_workspace_bytes(cache, s, hq)
    o = torch.full((q.numel() + 2 * guard,), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((2 * hq * s + 2 * guard,), 7.0, dtype=torch.float32, device="cuda")
    ws = torch.full((nbytes + 2 * guard,), 77, dtype=torch.uint8, device="cuda")
    K.paged_attention_forward(cache, q, i64([700 - s, 0]), i64([s, 0]), s, hq, 0.1, o[guard:], lse[guard:], ws[guard:])
    for t, n, v in ((o, q.numel(), 7.0), (lse, 2 * hq * s, 7.0), (ws, nbytes, 77)):
        assert (t[:guard] == v).all() and (t[guard + n:] == v).all()
    assert o[guard:-guard].isfinite().all() and (o[guard:-guard].view(2, -1)[1] == 0).all() and (lse[guard:-guard].view(2, -1)[1] == -np.inf).all()
    for t, u in zip((t for t in cache.tensors if t is not None), before):
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))


def test_a_cache_of_more_than_4_gib(K):
    """Pages on both sides of the 4 GiB mark, of both kinds of calls, against the same rows in a small cache."""
    hkv, dh, page = 8, 128, 64
    n_pages = (5 << 30) // (hkv * page * dh * 2)
    big = [torch.zeros((n_pages, hkv, page, dh), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ids = [n_pages - 1, 3, n_pages // 2, n_pages - 7, 11]
    small = [torch.randn((5, hkv, page, dh), device="cuda").bfloat16() for _ in range(2)]
    for x, y in zip(big, small):
        x[ids] = y
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    for s in (1, 100):
        q = torch.randn((1, s, 32, dh), device="cuda").bfloat16()
        got = run(K, K.KVCache.of(*big, table), q, [300 - s], None, 32, 0.09)
        ref = run(K, K.KVCache.of(*small, torch.arange(5, dtype=torch.int32, device="cuda")[None]), q, [300 - s], None, 32, 0.09)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("hq", [1, 64])
def test_the_longest_row(K, hq):
    """2^31 - 4096 tokens, all pages of the table the same one: what one page gives, and as often as it is there.  A lane adds up to 2^18 weights (1 at the
    most) in fp32: the sum, which grows evenly, is off by at most 2^18 / 2 roundings of 2^-24 of it, 2^-7, and so is the lse; the products' sums
    have 2^17 additions or fewer; weights and result are rounded to bf16."""
    dh, page, columns = 32, 4096, (1 << 19) - 1
    rng = np.random.default_rng(hq)
    k, v, q = bits(rng, (1, 1, page, dh)), bits(rng, (1, 1, page, dh), mean=1.0), bits(rng, (1, 1, hq, dh))
    cache = K.KVCache.of(dev_bf16(k), dev_bf16(v), torch.zeros((1, columns), dtype=torch.int32, device="cuda"))
    o, lse = run(K, cache, dev_bf16(q), [page * columns - 1], None, hq, dh ** -0.5)
    ref_o, ref_lse, mag, _ = og.attention({"k": si.bf16_bits_to_f64(k), "v": si.bf16_bits_to_f64(v), "page_table": np.zeros((1, 1), np.int64)},
                                          si.bf16_bits_to_f64(q), [page - 1], None, dh ** -0.5)
    assert np.abs(host_f64(o) - ref_o).max() <= ((2.0 ** -7 + 2.0 ** -7 + 2.0 ** -8 + 2.0 ** -7) * mag).max()
    assert np.abs(host_f64(lse) - ref_lse - np.log(columns)).max() <= 2.0 ** -7 + 2.0 ** -18


def ragged(rng, batch, longest, s, empty=True):
    """(tokens before, new tokens) of each row, some with none."""
    start, n = [int(x) for x in rng.integers(0, longest - s, batch)], [int(x) for x in rng.integers(0 if empty else 1, s + 1, batch)]
    start[0], n[0], n[-1] = longest - s, s, 0 if empty else s
    return start, n


# batch, longest row, seq, query and KV heads, head_dim, page: more rows than are put in order, and fewer; keys cut into parts or not; 16, 32 and 128 rows to a workgroup
RAGGED = [(70, 200, 1, 4, 2, 32, 16), (3, 3000, 2, 16, 8, 64, 16), (9, 1500, 1, 2, 1, 128, 32), (2, 5000, 3, 16, 2, 128, 128), (66, 150, 9, 4, 1, 32, 16), (5, 900, 40, 8, 8, 64, 16),
          (2, 2600, 70, 4, 2, 128, 64), (1, 4500, 33, 4, 1, 32, 256), (70, 80, 34, 8, 8, 128, 16)]


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("case", RAGGED, ids=str)
def test_ragged_batches(K, case, e4m3):
    batch, longest, s, hq, hkv, dh, page = case
    rng = np.random.default_rng(batch + longest + e4m3)
    start, n = ragged(rng, batch, longest, s, empty=batch > 1)
    pages = Pages(rng, [a + m for a, m in zip(start, n)], hkv, dh, page, e4m3, columns=-(-longest // page) + 3)
    qb = bits(rng, (batch, s, hq, dh), 2.0)
    o, lse = run(K, pages.device(K), spoiled(dev_bf16(qb), n), start, n, hq, dh ** -0.5)
    check(o, lse, og.attention(pages.oracle(), si.bf16_bits_to_f64(qb), start, n, dh ** -0.5), dh)


def test_many_rows_of_an_e4m3_cache(K):
    """Eight waves to a workgroup: rows and keys that end inside its tiles, NaN among the last tokens, a page that does not exist; sampled rows against the oracle."""
    rng = np.random.default_rng(9)
    b, s, hq, hkv, dh, page = 4, 530, 64, 8, 128, 16
    start, n = [300, 0, 77, 5], [530, 17, 399, 0]
    pages = Pages(rng, [a + m for a, m in zip(start, n)], hkv, dh, page, True)
    pages.table[2, 3] = -1
    qb = bits(rng, (b, s, hq, dh), 2.0)
    p = start[0] + 500
    pages.codes[1][pages.table[0, p // page], 3, p % page, 100] = 0x7F
    o, lse = run(K, pages.device(K), spoiled(dev_bf16(qb), n), start, n, hq, 0.088)
    assert torch.isnan(o[0, 500:, 24:32, 100]).all() and int(torch.isnan(o).sum()) == 30 * 8
    o[0, 500:, 24:32, 100] = 0
    cache, got, q = pages.oracle(), host_f64(o), si.bf16_bits_to_f64(qb)
    cache["v"] = np.nan_to_num(cache["v"], nan=0.0)
    for i in range(b):
        assert np.all(got[i, n[i]:] == 0) and bool(torch.isneginf(lse[i, :, n[i]:]).all())
        for t in sorted({0, 1, 31, 32, 33, 63, 64, 127, 200, n[i] - 1} & set(range(n[i]))):
            one = dict(cache, page_table=cache["page_table"][i:i + 1])
            heads = [0, 9, 31, 63]
            for h in heads:
                j = h // (hq // hkv)
                sub = {"k": one["k"][:, j:j + 1], "v": one["v"][:, j:j + 1], "page_table": one["page_table"]}
                ref = og.attention(sub, q[i:i + 1, t:t + 1, h:h + 1], [start[i] + t], None, 0.088)
                if i == 0 and t >= 500 and j == 3:
                    ref[0][..., 100], got[i, t, h, 100] = 0, 0
                check(torch.from_numpy(got[i:i + 1, t:t + 1, h:h + 1]), lse[i:i + 1, h:h + 1, t:t + 1], ref, dh)


@pytest.mark.parametrize("s,hq,longest", [(1, 4, 3000), (7, 4, 3000), (60, 4, 3000), (60, 16, 200)])
def test_missing_pages_and_parts(K, s, hq, longest):
    """Whole parts of a row's keys lie in pages that do not exist, or single pages of each."""
    rng = np.random.default_rng(s)
    start = [longest - s, longest - s, longest // 2]
    pages = Pages(rng, [a + s for a in start], 2, 64, 16, s == 7)
    pages.table[0, 10:100] = -1
    pages.table[1, rng.integers(0, pages.table.shape[1], 60)] = 1 << 20
    pages.table[2, :20] = -7
    qb = bits(rng, (3, s, hq, 64), 2.0)
    o, lse = run(K, pages.device(K), dev_bf16(qb), start, None, hq, 0.125)
    check(o, lse, og.attention(pages.oracle(), si.bf16_bits_to_f64(qb), start, None, 0.125), 64)


@pytest.mark.parametrize("s,group,e4m3", [(2, 8, True), (20, 1, True), (10, 3, False), (150, 1, True), (100, 8, True), (130, 2, False)])
def test_many_values_that_are_not_finite(K, s, group, e4m3):
    """NaN and infinities strewn over the new tokens' keys and values: every element is NaN exactly where a token sees one that it depends on."""
    rng = np.random.default_rng(s + group)
    hkv, dh, start = 2, 64, 40
    pages = Pages(rng, [start + s], hkv, dh, 16, e4m3)
    qb = bits(rng, (1, s, group * hkv, dh), 2.0)
    clean, clean_lse = run(K, pages.device(K), dev_bf16(qb), [start], None, group * hkv, 0.125)
    odd_v, odd_k = np.full((hkv, dh), 10 ** 9), np.full(hkv, 10 ** 9)            # the first position of each
    for _ in range(12):
        t, j, d, w = int(rng.integers(s)), int(rng.integers(hkv)), int(rng.integers(dh)), int(rng.integers(4) > 0)
        p = start + t
        pages.codes[w][pages.table[0, p // 16], j, p % 16, d] = 0x7F if e4m3 else (0x7FC0 if rng.integers(2) else 0xFF80)
        if w:
            odd_v[j, d] = min(odd_v[j, d], p)
        else:
            odd_k[j] = min(odd_k[j], p)
    o, lse = run(K, pages.device(K), dev_bf16(qb), [start], None, group * hkv, 0.125)
    o, clean = host_f64(o)[0], host_f64(clean)[0]
    p = start + np.arange(s)[:, None, None]
    # an infinite key makes a score of either sign of infinity, or NaN: with +infinity and NaN the token has no result, with -infinity the key has no weight
    for h in range(group * hkv):
        j = h // group
        by_v, by_k = p[:, 0] >= odd_v[j], (p[:, 0] >= odd_k[j]) & np.ones((s, dh), bool)
        assert np.all(~np.isfinite(o[:, h])[by_v & ~by_k])
        untouched = ~by_v & ~by_k
        assert np.array_equal(o[:, h][untouched], clean[:, h][untouched])
        rows = ~by_k[:, 0]
        assert torch.equal(lse[0, h].cpu()[rows], clean_lse[0, h].cpu()[rows])


# tokens, heads of a group, KV heads, head_dim, e4m3: one, few and many rows of a KV head, and eight waves to a workgroup
BAD_KEYS = [(1, 4, 2, 64, True), (1, 4, 2, 128, False), (6, 4, 2, 64, True), (20, 1, 2, 32, True), (30, 3, 2, 64, True), (70, 4, 2, 128, True), (150, 1, 2, 64, False), (130, 8, 64, 128, True)]


@pytest.mark.parametrize("longest", [50, 1500])
@pytest.mark.parametrize("case", BAD_KEYS, ids=str)
def test_a_key_that_is_nan_leaves_no_result_where_it_is_seen(K, case, longest):
    """NaN in one element of a key, before the call's tokens or among them: every token that sees the key has NaN for its whole result and its statistic, every
    other token, and every other KV head, what the oracle has."""
    s, group, hkv, dh, e4m3 = case
    rng = np.random.default_rng(s + longest)
    start, hq = longest, group * hkv
    if hkv > 2:
        start = 40                                        # the oracle's time
    pages = Pages(rng, [start + s], hkv, dh, 16, e4m3)
    bad = [(0, start + s // 2), (1, start // 3)]          # KV head, position
    for j, p in bad:
        pages.codes[0][pages.table[0, p // 16], j, p % 16, int(rng.integers(dh))] = 0xFF if e4m3 else 0x7FC1
    qb = bits(rng, (1, s, hq, dh), 2.0)
    o, lse = run(K, pages.device(K), dev_bf16(qb), [start], None, hq, dh ** -0.5)
    o, lse = host_f64(o), host_f64(lse)
    p = start + np.arange(s)
    for j, at in bad:
        sees = p >= at
        heads = slice(j * group, (j + 1) * group)
        assert np.isnan(o[0, sees][:, heads]).all() and np.isnan(lse[0, heads][:, sees]).all() and sees.any()
        o[0][np.ix_(sees, range(j * group, (j + 1) * group))] = 0
        lse[0][np.ix_(range(j * group, (j + 1) * group), sees)] = 0
    cache, q = pages.oracle(), si.bf16_bits_to_f64(qb)
    for h in range(0, hq, max(1, hq // 8)):
        j = h // group
        one = {"k": cache["k"][:, j:j + 1], "v": cache["v"][:, j:j + 1], "page_table": cache["page_table"]}
        ref = og.attention(one, q[:, :, h:h + 1], [start], None, dh ** -0.5)
        nan = np.isnan(ref[1])
        assert np.array_equal(np.isnan(ref[0]).all(-1)[0, :, 0], nan[0, 0]) and (not nan.any() or j < 2)
        ref = [np.where(np.isnan(x), 0.0, x) for x in ref]
        check(torch.from_numpy(o[:, :, h:h + 1]), torch.from_numpy(lse[:, h:h + 1]), ref, dh)
