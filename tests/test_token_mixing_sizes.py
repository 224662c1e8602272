"""Workspace sizes and limits of the norm of queries and keys and of linear attention, on the host (no GPU needed)."""
import pytest


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def _never_falls(sizes, what):
    assert all(s > 0 for s in sizes), what
    assert all(a <= b for a, b in zip(sizes, sizes[1:])), f"{what}: {sizes}"


LENGTHS = [1, 2, 3, 63, 64, 65, 127, 128, 500, 900, 1000, 1100, 1400, 2047, 2048, 4096, 4097, 8192, 65536, 10 ** 6]


@pytest.mark.parametrize("Hq,Hkv,dh", [(1, 1, 32), (12, 12, 64), (8, 1, 64), (18, 6, 32), (32, 8, 128)])
def test_scratch_serves_smaller_batches_and_sequences(K, Hq, Hkv, dh):
    for query in (K.qk_norm_rope_backward_workspace_bytes, K.linear_attention_workspace_bytes, K.linear_attention_backward_workspace_bytes):
        for B in (1, 3, 40, 600):
            _never_falls([query(B, S, Hq, Hkv, dh) for S in LENGTHS], f"{query.__name__}: seq at B = {B}")
        for S in (1, 130, 4096):
            _never_falls([query(B, S, Hq, Hkv, dh) for B in range(1, 200)], f"{query.__name__}: batch at S = {S}")
    assert K.qk_norm_rope_backward_workspace_bytes(64, 8192, Hq, Hkv, dh) <= 8 * dh * 1024
    # nothing that a caller of one row and a few tokens would mind: a state for each 64 of them
    assert K.linear_attention_workspace_bytes(1, 65, Hq, Hkv, dh) == 2 * Hkv * dh * dh * 4


def test_sizes_that_no_launch_holds_are_rejected(K):
    most = 1 << 22
    assert K.linear_attention_workspace_bytes(most - 1, 1, 1, 1, 32) > 0
    for query in (K.linear_attention_workspace_bytes, K.linear_attention_backward_workspace_bytes):
        assert query(most, 1, 1, 1, 32) == 0 and query(most // 4, 1, 4, 4, 32) == 0
        assert query(1, 1 << 30, 1, 1, 32) == 0 and query(1, 64, 65536, 1, 32) == 0
    assert K.qk_norm_rope_backward_workspace_bytes(1 << 31, 1, 1, 1, 32) == 0
    with pytest.raises(K.DLayerError, match="too large"):
        K.linear_attention_step(None, None, None, None, None, None, most, 1, 1, 32, 1.0, None, stream=0)
