"""Buffers of linear attention that overlap where a call would read what another part of it has written: turned down before anything is launched
(on the host, with addresses that nothing looks behind: every call here has to be rejected for its addresses alone)."""
import pytest

B, S, HQ, HKV, DH = 2, 100, 4, 2, 64
QUERIES, KEYS, STATES = B * S * HQ * DH * 2, B * S * HKV * DH * 2, B * HKV * DH * DH * 4


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def _apart():
    """Addresses far from one another."""
    names = ("q", "k", "v", "log", "s_in", "d_o", "ds_out", "o", "s_out", "dq", "dk", "dv", "ds_in", "ws")
    return {n: (i + 1) << 32 for i, n in enumerate(names)}


def _refused(K, name, *args):
    from paper_2602_08387_amd import binding
    rc = getattr(binding.lib, name)(*args)
    message = binding.lib.dlayer_last_error().decode()
    assert rc == -1 and "overlap" in message, (name, rc, message)


@pytest.mark.parametrize("where", ["q", "k", "v"])
@pytest.mark.parametrize("end", [False, True])
def test_output_over_an_input(K, where, end):
    size = QUERIES if where == "q" else KEYS
    a = dict(_apart())
    a["o"] = a[where] + size - 16 if end else a[where]      # on it, or over its last bytes
    _refused(K, "linear_attention_forward", a["q"], a["k"], a["v"], a["log"], None, a["s_in"], B, S, HQ, HKV, DH, 1.0, a["o"], a["s_out"], a["ws"], None)
    # one token of every row
    size //= S
    a["o"] = a[where] + size - 16 if end else a[where]
    _refused(K, "linear_attention_step", a["q"], a["k"], a["v"], a["log"], None, a["s_in"], B, HQ, HKV, DH, 1.0, a["o"], None)


@pytest.mark.parametrize("output", ["dq", "dk", "dv"])
@pytest.mark.parametrize("where", ["q", "k", "v", "d_o"])
def test_gradient_over_an_input(K, output, where):
    for end in (False, True):
        a = _apart()
        a[output] = a[where] + (QUERIES if where in ("q", "d_o") else KEYS) - 16 if end else a[where]
        _refused(K, "linear_attention_backward", a["q"], a["k"], a["v"], a["log"], None, a["s_in"], a["d_o"], a["ds_out"], B, S, HQ, HKV, DH, 1.0,
                 a["dq"], a["dk"], a["dv"], a["ds_in"], a["ws"], None)


def test_gradient_of_a_state_over_the_state(K):
    """dq is formed from state_in while d_state_in is written."""
    for shift in (0, 16, STATES - 16, 16 - STATES):
        a = _apart()
        a["ds_in"] = a["s_in"] + shift
        _refused(K, "linear_attention_backward", a["q"], a["k"], a["v"], a["log"], None, a["s_in"], a["d_o"], a["ds_out"], B, S, HQ, HKV, DH, 1.0,
                 a["dq"], a["dk"], a["dv"], a["ds_in"], a["ws"], None)


def test_states_in_part_over_one_another(K):
    """In place is fine, shifted is not."""
    for shift in (16, STATES - 16, 16 - STATES):
        a = _apart()
        _refused(K, "linear_attention_forward", a["q"], a["k"], a["v"], a["log"], None, a["s_in"], B, S, HQ, HKV, DH, 1.0, a["o"], a["s_in"] + shift, a["ws"], None)
        _refused(K, "linear_attention_backward", a["q"], a["k"], a["v"], a["log"], None, a["s_in"], a["d_o"], a["ds_out"], B, S, HQ, HKV, DH, 1.0,
                 a["dq"], a["dk"], a["dv"], a["ds_out"] + shift, a["ws"], None)
