"""Arguments that the paged cache, the attention over it and the log-probabilities turn down, and their size queries, on the host: addresses that nothing
looks behind, every call has to be rejected before anything is launched."""
import ctypes as C

import pytest

B, S, HQ, HKV, DH, PAGE, PAGES, COLUMNS = 3, 20, 8, 2, 64, 16, 12, 4


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def cache(K, **changes):
    c = K.KVCache(1 << 32, 2 << 32, 3 << 32, 4 << 32, 5 << 32, PAGES, HKV, PAGE, DH, B, COLUMNS, K.DLAYER_CACHE_E4M3)
    for n, x in changes.items():
        setattr(c, n, x)
    return c


def refused(K, name, *args):
    from paper_2602_08387_amd import binding
    rc = getattr(binding.lib, name)(*args)
    message = binding.lib.dlayer_last_error().decode()
    assert rc == -1 and message.startswith(name), (name, rc, message)
    return message


BAD_CACHES = [dict(n_pages=0), dict(n_kv_heads=0), dict(batch=0), dict(max_pages=0), dict(max_pages=-1), dict(head_dim=96), dict(head_dim=256), dict(page_size=8), dict(page_size=24),
              dict(page_size=8192), dict(page_size=0), dict(dtype=2), dict(dtype=-1), dict(max_pages=1 << 27), dict(k=0), dict(v=0), dict(k=(1 << 32) + 8), dict(page_table=0),
              dict(v=(1 << 32) + 16), dict(k_scale=0), dict(v_scale=(4 << 32) + 4), dict(dtype=0)]
A = [(i + 10) << 32 for i in range(8)]        # addresses far from one another and from the cache


@pytest.mark.parametrize("changes", BAD_CACHES, ids=str)
def test_caches(K, changes):
    c = C.byref(cache(K, **changes))
    refused(K, "kv_cache_append", c, A[0], A[1], A[2], None, None, S, HQ, 1e4, 0, A[3], None)
    refused(K, "kv_cache_read", c, None, None, S, A[0], A[1], None)
    refused(K, "paged_attention_forward", c, A[0], None, None, S, HQ, 0.1, A[1], None, A[2], None)


@pytest.mark.parametrize("page", [16, 4096])
def test_the_longest_row(K, page):
    """A row's keys, filled up to whole tiles of at most 128, are counted in 32 bits."""
    columns = ((1 << 31) - 4096) // page
    assert K.paged_attention_workspace_bytes(cache(K, page_size=page, max_pages=columns), 1, HKV) > 0
    assert K.paged_attention_workspace_bytes(cache(K, page_size=page, max_pages=columns + 1), 1, HKV) == 0
    c = C.byref(cache(K, page_size=page, max_pages=columns + 1))
    assert "2^31" in refused(K, "paged_attention_forward", c, A[0], None, None, S, HQ, 0.1, A[1], None, A[2], None)


def test_append(K):
    c = C.byref(cache(K))
    call = lambda *a: refused(K, "kv_cache_append", *a, None)  # noqa: E731
    call(None, A[0], A[1], A[2], None, None, S, HQ, 1e4, 0, A[3])
    call(c, A[0], None, A[2], None, None, S, HQ, 1e4, 0, A[3])
    call(c, A[0], A[1], A[2] + 2, None, None, S, HQ, 1e4, 0, A[3])
    call(c, A[0], A[1], A[2], None, None, 0, HQ, 1e4, 0, A[3])
    call(c, A[0], A[1], A[2], None, None, S, HQ, 1e4, 0, None)              # q without q_out
    call(c, None, A[1], A[2], None, None, S, HQ, 1e4, 0, A[3])
    call(c, A[0], A[1], A[2], None, None, S, HQ, 0.0, 0, A[3])              # q, but no rotation
    call(c, A[0], A[1], A[2], None, None, S, 0, 1e4, 0, A[3])
    call(c, A[0], A[1], A[2], None, None, S, HQ, -1.0, 0, A[3])
    call(c, A[0], A[1], A[2], None, None, S, HQ, float("nan"), 0, A[3])
    call(c, A[0], A[1], A[2], None, None, S, HQ, float("inf"), 0, A[3])
    call(c, A[0], A[1], A[2], None, None, S, HQ, 1e4, 2, A[3])
    size = B * S * HQ * DH * 2
    assert "overlap" in call(c, A[0], A[1], A[2], None, None, S, HQ, 1e4, 0, A[0] + 16)
    assert "overlap" in call(c, A[0], A[0] + size - 16, A[2], None, None, S, HQ, 1e4, 0, A[0])
    for part, held in ((1, PAGES * HKV * PAGE * DH), (2, PAGES * HKV * PAGE * DH), (3, PAGES * HKV * PAGE), (5, B * COLUMNS * 4)):
        at = (part << 32) + held - 16
        assert "overlap" in call(c, A[0], at, A[2], None, None, S, HQ, 1e4, 0, A[3])
        assert "overlap" in call(c, A[0], A[1], at, None, None, S, HQ, 1e4, 0, A[3])
        assert "overlap" in call(c, A[0], A[1], A[2], None, None, S, HQ, 1e4, 0, at)


def test_read(K):
    c = C.byref(cache(K))
    call = lambda *a: refused(K, "kv_cache_read", *a, None)  # noqa: E731
    call(c, None, None, S, None, A[1])
    call(c, None, None, S, A[0], A[1] + 8)
    call(c, None, None, 0, A[0], A[1])
    assert "overlap" in call(c, None, None, S, A[0], A[0] + 16)
    assert "overlap" in call(c, None, None, S, 2 << 32, A[1])


def test_attention(K):
    c = C.byref(cache(K))
    call = lambda *a: refused(K, "paged_attention_forward", *a, None)  # noqa: E731
    call(c, None, None, None, S, HQ, 0.1, A[1], A[3], A[2])
    call(c, A[0], None, None, S, HQ, 0.1, None, A[3], A[2])
    call(c, A[0], None, None, S, HQ, 0.1, A[1], A[3], None)
    call(c, A[0], None, None, S, 7, 0.1, A[1], A[3], A[2])
    call(c, A[0], None, None, S, 0, 0.1, A[1], A[3], A[2])
    call(c, A[0], None, None, 1 << 28, HQ, 0.1, A[1], A[3], A[2])
    many = C.byref(cache(K, batch=1 << 23, max_pages=1))                      # more workgroups than a launch holds
    call(many, A[0], None, None, 1, 4, 0.1, A[1], A[3], A[2])
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        call(c, A[0], None, None, S, HQ, scale, A[1], A[3], A[2])
    assert "overlap" in call(c, A[0], None, None, S, HQ, 0.1, A[0], A[3], A[2])
    assert "overlap" in call(c, A[0], None, None, S, HQ, 0.1, 1 << 32, A[3], A[2])


def test_logprobs(K):
    T, V, ld, n = 5, 1001, 1008, 4
    call = lambda *a: refused(K, "token_logprobs_forward", *a, None)  # noqa: E731
    good = [A[0], A[1], T, V, ld, 1.0, n, A[2], A[3], A[4], A[5], A[6], A[7]]
    for i, x in ((0, None), (0, A[0] + 2), (2, 0), (2, 1 << 22), (3, 0), (3, ld + 1), (4, 1004), (4, 1 << 24), (5, 0.0), (5, -1.0), (5, float("nan")), (5, float("inf")), (6, -1),
                 (6, 65), (6, 0), (1, None), (12, None)):
        bad = list(good)
        bad[i] = x
        call(*bad)
    call(A[0], A[1], T, 3, 8, 1.0, 4, *good[7:])                            # more alternatives than tokens
    call = lambda *a: refused(K, "token_logprobs_backward", *a, None)  # noqa: E731
    good = [A[0], A[1], A[2], A[3], A[4], A[5], T, V, ld, 1.0, A[6]]
    for i, x in ((0, None), (2, None), (3, None), (1, None), (6, 0), (7, 0), (8, V), (9, 0.0), (10, None), (10, A[0] + 16)):
        bad = list(good)
        bad[i] = x
        call(*bad)
    call(A[0], A[1], A[2], A[3], None, None, T, V, ld, 1.0, A[6])
    call(A[0], A[1], A[2], A[3], A[4], A[5], (1 << 22) - 1, 40000, 40000, 1.0, A[0])


def test_memory_in_common(K):
    """Buffers that a call would write to while others of its workgroups read them."""
    held, scales, table = PAGES * HKV * PAGE * DH, PAGES * HKV * PAGE, B * COLUMNS * 4
    for changes in (dict(v_scale=4 << 32, k_scale=(4 << 32) + 16), dict(k_scale=1 << 32), dict(v_scale=(2 << 32) + held - 16), dict(k_scale=(1 << 32) - scales + 16),
                    dict(page_table=(2 << 32) + 64), dict(page_table=(4 << 32) + scales - 4), dict(k=(5 << 32) + table - 16)):
        assert "overlap" in refused(K, "kv_cache_read", C.byref(cache(K, **changes)), None, None, S, A[0], A[1], None), changes
    c, of_q = C.byref(cache(K)), B * S * HQ * DH * 2
    for lse in (A[0] + of_q - 4, A[1], (1 << 32) + 4, (5 << 32) + 4, A[1] - 4):
        assert "overlap" in refused(K, "paged_attention_forward", c, A[0], None, None, S, HQ, 0.1, A[1], lse, A[2], None)
    T, V, ld, n = 5, 1001, 1008, 4
    for i in range(5):
        for at in (A[0] + T * ld * 2 - 4, A[1] + T * 8 - 8):
            out = list(A[2:7])
            out[i] = at
            assert "overlap" in refused(K, "token_logprobs_forward", A[0], A[1], T, V, ld, 1.0, n, *out, A[7], None)
    for i in range(1, 6):
        inputs = list(A[:6])
        inputs[i] = A[6] + 8
        assert "overlap" in refused(K, "token_logprobs_backward", *inputs, T, V, ld, 1.0, A[6], None)


def test_factors_whose_exponents_would_overflow(K):
    assert "1e30" in refused(K, "paged_attention_forward", C.byref(cache(K)), A[0], None, None, S, HQ, 3e38, A[1], A[3], A[2], None)
    assert "1e30" in refused(K, "token_logprobs_forward", A[0], A[1], 5, 1001, 1008, 3e38, 4, *A[2:7], A[7], None)
    assert "1e30" in refused(K, "token_logprobs_backward", *A[:6], 5, 1001, 1008, 3e38, A[6], None)


def test_workspaces_do_not_fall(K):
    size = lambda s=S, hq=HQ, **ch: K.paged_attention_workspace_bytes(cache(K, k=0, v=0, page_table=0, **ch), s, hq)  # noqa: E731
    for field, values in (("batch", (1, 2, 7, 8, 64, 65, 511, 512, 513, 4000)), ("max_pages", (1, 2, 3, 15, 16, 17, 100, 5000))):
        for s in (1, 2, 4, 5, 16, 17, 33, 300):
            got = [size(s, **{field: x}) for x in values]
            assert got == sorted(got) and got[0] > 0
    for batch in (1, 3, 100):
        for columns in (1, 64, 4096):
            got = [size(s, batch=batch, max_pages=columns) for s in (1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 1000, 10000)]
            assert got == sorted(got)
    assert size(hq=7) == 0 and size(0) == 0 and size(head_dim=48) == 0
    size = K.token_logprobs_workspace_bytes
    for n in (0, 1, 64):
        for V in (1000, 4096, 4097, 128256):
            got = [size(T, V, n) for T in (1, 2, 3, 9, 100, 1023, 1024, 1025, 1 << 20)]
            assert got == sorted(got) and 0 < got[0] and got[-1] <= 528 << 10
        for T in (1, 5, 700, 5000):
            got = [size(T, V, n) for V in (64, 4095, 4096, 4097, 8192, 8193, 50257, 128256, 1 << 23)]
            assert got == sorted(got)
    assert size(0, 10) == 0 and size(4, 10, 11) == 0 and size(4, 100, 65) == 0


def test_handles_of_tensors_that_do_not_fit(K):
    import torch
    t = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype)  # noqa: E731
    table, k = t(2, 4, dtype=torch.int32), t(3, 2, 16, 64)
    codes, scale = t(3, 2, 16, 64, dtype=torch.uint8), t(3, 2, 16, dtype=torch.uint8)
    for args in ((k, t(3, 2, 16, 32), table), (k, k.float(), table), (k.float(), k.float(), table), (k[0], k[0], table), (k, k, table.long()), (k, k, table[0]),
                 (codes, codes, table), (codes, codes, table, scale), (k, k, table, scale, scale), (codes, codes, table, scale, scale[:2]),
                 (codes, codes, table, scale, scale.int())):
        with pytest.raises(K.DLayerError, match="KVCache"):
            K.KVCache.of(*args)
    with pytest.raises(K.DLayerError, match="GPU"):
        K.KVCache.of(k, k, table)


def test_workspaces_in_common(K):
    """A workspace that lies over what the call reads or writes, at either end."""
    c, of_q, of_rows = cache(K), B * S * HQ * DH * 2, B * 8
    bytes_ = K.paged_attention_workspace_bytes(c, S, HQ)
    for at, size in ((A[0], of_q), (A[1], of_q), (A[3], B * S * HQ * 4), (A[4], of_rows), (A[5], of_rows), (1 << 32, PAGES * HKV * PAGE * DH), (2 << 32, PAGES * HKV * PAGE * DH),
                     (3 << 32, PAGES * HKV * PAGE), (4 << 32, PAGES * HKV * PAGE), (5 << 32, B * COLUMNS * 4)):
        for ws in (at - bytes_ // 16 * 16 + 16, (at + size - 1) // 16 * 16):
            assert "workspace" in refused(K, "paged_attention_forward", C.byref(c), A[0], A[4], A[5], S, HQ, 0.1, A[1], A[3], ws, None), (hex(at), hex(ws))
    T, V, ld, n = 5, 10001, 10008, 4
    bytes_ = K.token_logprobs_workspace_bytes(T, V, n)
    for at, size in ((A[0], T * ld * 2), (A[1], T * 8), (A[2], T * 4), (A[3], T * 4), (A[4], T * 4), (A[5], T * n * 8), (A[6], T * n * 4)):
        for ws in (at - bytes_ // 16 * 16 + 16, (at + size - 1) // 16 * 16):
            assert "workspace" in refused(K, "token_logprobs_forward", A[0], A[1], T, V, ld, 1.0, n, *A[2:7], ws, None), (hex(at), hex(ws))


def test_results_in_common(K):
    """Any two of the log-probabilities' results, the second at either end of the first."""
    T, V, ld, n = 5, 1001, 1008, 4
    sizes = [T * 4, T * 4, T * 4, T * n * 8, T * n * 4]
    for i in range(5):
        for j in range(5):
            for at in (A[2 + i], A[2 + i] + sizes[i] - 4, A[2 + i] - sizes[j] + 4):
                out = list(A[2:7])
                out[j] = at
                if i != j:
                    assert "overlap" in refused(K, "token_logprobs_forward", A[0], A[1], T, V, ld, 1.0, n, *out, A[7], None), (i, j)


def test_rows_places_in_common(K):
    """start and lengths under what a call writes."""
    c, of_q, of_kv, rows = C.byref(cache(K)), B * S * HQ * DH * 2, B * S * HKV * DH * 2, B * 8
    held, scales = PAGES * HKV * PAGE * DH, PAGES * HKV * PAGE
    for at, size in ((A[3], of_q), (1 << 32, held), (2 << 32, held), (3 << 32, scales), (4 << 32, scales)):
        for x in (at - rows + 8, at + size - 8):
            for places in ((x, None), (None, x)):
                assert "overlap" in refused(K, "kv_cache_append", c, A[0], A[1], A[2], *places, S, HQ, 1e4, 0, A[3], None), hex(x)
    for at, size in ((A[0], of_kv), (A[1], of_kv)):
        for x in (at - rows + 8, at + size - 8):
            for places in ((x, None), (None, x)):
                assert "overlap" in refused(K, "kv_cache_read", c, *places, S, A[0], A[1], None), hex(x)
    for at, size in ((A[1], of_q), (A[3], B * S * HQ * 4)):
        for x in (at - rows + 8, at + size - 8):
            for places in ((x, None), (None, x)):
                assert "overlap" in refused(K, "paged_attention_forward", c, A[0], *places, S, HQ, 0.1, A[1], A[3], A[2], None), hex(x)


def test_tensors_of_other_types(K):
    """A tensor of a narrower type than the call reads or writes ends before the call does: each tensor in turn, before any address is looked at."""
    import torch
    i64, f32, bf16 = (torch.empty(8, dtype=t) for t in (torch.int64, torch.float32, torch.bfloat16))
    c = cache(K)
    calls = ((K.kv_cache_append, (c, bf16, bf16, bf16, i64, i64, S, HQ, 1e4, 0, bf16), ("q", "k", "v", "start", "lengths", "q_out")),
             (K.kv_cache_read, (c, i64, i64, S, bf16, bf16), ("start", "lengths", "k", "v")),
             (K.paged_attention_forward, (c, bf16, i64, i64, S, HQ, 0.1, bf16, f32, bf16), ("q", "start", "lengths", "o", "lse")),
             (K.token_logprobs_forward, (bf16, i64, 5, 1001, 1008, 1.0, 4, f32, f32, f32, i64, f32, bf16),
              ("logits", "targets", "logprobs", "entropy", "lse", "top_ids", "top_logprobs")),
             (K.token_logprobs_backward, (bf16, i64, f32, f32, f32, f32, 5, 1001, 1008, 1.0, bf16),
              ("logits", "targets", "lse", "entropy", "d_logprobs", "d_entropy", "dlogits")))
    narrower = {torch.int64: torch.int32, torch.float32: torch.bfloat16, torch.bfloat16: torch.uint8}
    for call, good, names in calls:
        at = [i for i, x in enumerate(good) if isinstance(x, torch.Tensor)][:len(names)]
        for i, name in zip(at, names):
            # the others are left out, so that nothing but this one's type is to be refused
            args = [None if j in at and j != i else x for j, x in enumerate(good)]
            args[i] = torch.empty(8, dtype=narrower[good[i].dtype])
            with pytest.raises(K.DLayerError, match=f"^{name} must be"):
                call(*args)
