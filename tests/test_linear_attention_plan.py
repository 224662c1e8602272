"""How linear attention cuts its work, on the host, and that the cases of test_gpu_linear_attention_paths take every way there is."""
import pytest

from tests.test_gpu_linear_attention_paths import CASES


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def _ways(K, B, S, Hq, Hkv, dh, backward):
    chunks, segments, parts = K.linear_attention_plan(B, S, Hq, Hkv, dh, backward)
    total, group = -(-S // 64), Hq // Hkv
    assert (segments - 1) * chunks < total <= segments * chunks
    heads = -(-group // parts)
    assert heads * (parts - 1) < group                    # no part without a head
    ways = {"one segment" if segments == 1 else "segments"}
    if heads >= 2:
        ways.add("a pair of heads")
    if heads >= 4:
        ways.add("two pairs")
    if heads >= 3 and heads % 2:
        ways.add("a head left over from a pair")
    if parts > 1 and heads >= 2:
        ways.add("parts of several heads")
    if segments > 1 and chunks >= 8:
        ways.add("segments of many chunks")
    return ways


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("backward", [False, True])
def test_cases_take_every_way(K, dh, backward):
    ways = set().union(*(_ways(K, *c[:5], backward) for c in CASES if c[4] == dh))
    want = {"one segment", "segments", "a pair of heads", "a head left over from a pair", "segments of many chunks"}
    # a backward's parts are fewer, since other workgroups run beside them: its groups are whole in these cases
    want |= {"two pairs"} if backward else {"parts of several heads"}
    assert want <= ways, want - ways


def test_large_calls_take_the_ways_that_are_tested(K):
    """The layer of the 8B model over long sequences, and a long prompt."""
    for B, S, Hq, Hkv, backward in ((2, 8192, 32, 8, False), (2, 8192, 32, 8, True), (1, 65536, 16, 8, False)):
        ways = _ways(K, B, S, Hq, Hkv, 128, backward)
        tested = set().union(*(_ways(K, *c[:5], backward) for c in CASES if c[4] == 128))
        assert "segments" in ways and "a pair of heads" in ways
        assert ways <= tested, ways - tested


def test_bad_arguments(K):
    for bad in ((0, 64, 1, 1, 64), (1, 64, 3, 2, 64), (1, 64, 2, 2, 48)):
        with pytest.raises(K.DLayerError):
            K.linear_attention_plan(*bad)
    with pytest.raises(K.DLayerError, match="backward"):
        K.linear_attention_plan(1, 64, 2, 2, 64, backward=2)
