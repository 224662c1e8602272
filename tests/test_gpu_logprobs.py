"""Log-probabilities of tokens, entropies and likeliest tokens, and their gradient, through the C ABI against the fp64 oracle.

Tolerances.  A row's exponents t = z - max are formed in fp32: off by a few units of 2^-24 of t, and the sums of up to 2^18 terms in blocks are off by 2^-18 at the
very most; lse and log-probabilities by that and by their own rounding, 2^-23 of their parts' magnitude: 4e-6 + 3e-7 * (|z| + |max|).  Entropy = ln S - U / S, both at least 0 and
so no more than it: each is off by 2^-18 of itself, and ln S by some units of 2^-24 more, since S is 1 and a little in a row that is all but certain and every addition to it rounds
by as much; either way, so that four are allowed for.  1e-5 * entropy + 2.5e-7.  Gradient: p is off by 2^-24 of |z| + |lse| and a few units, its products round, then one rounding to bf16
(2^-8 of the value), of a sum whose two terms at the target may cancel: 2^-8 |d| + 4e-6 * (1 + |z| + |lse|) of the terms' magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import generation as og
from synth import inputs as si
from tests.paged import garbage, workspace
from tests.parity import dev_bf16, host_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    import paper_2602_08387_amd as k
    return k


def forward(K, logits, targets, V, inverse=1.0, n_top=0, stream=None):
    T, ld = logits.shape
    out = [garbage((T,), torch.float32) if targets is not None else None, garbage((T,), torch.float32), garbage((T,), torch.float32)]
    out += [torch.full((T, n_top), -77, dtype=torch.int64, device="cuda"), garbage((T, n_top), torch.float32)] if n_top else [None, None]
    ws = workspace(K.token_logprobs_workspace_bytes(T, V, n_top))
    K.token_logprobs_forward(logits, targets, T, V, ld, inverse, n_top, *out, ws, stream)
    return out


def check(got, z, targets, inverse, n_top):
    ref = og.logprobs(z, targets, inverse, n_top)
    size = np.max(np.abs(np.where(np.isfinite(z), z, 0.0)), axis=-1) * inverse
    tol = 4e-6 + 6e-7 * size
    for g, r in ((got[0], ref[0]), (got[2], ref[2])):
        if g is not None:
            g = host_f64(g)
            fine = np.isfinite(r)
            assert np.array_equal(g[~fine], r[~fine])
            assert np.all(np.abs(g - r)[fine] <= tol[fine]), np.max((np.abs(g - r) / tol)[fine])
    h = host_f64(got[1])
    assert np.all(np.abs(h - ref[1]) <= 1e-5 * ref[1] + 2.5e-7), np.max(np.abs(h - ref[1]))
    if n_top:
        assert np.array_equal(got[3].cpu().numpy(), ref[3])
        g, r = host_f64(got[4]), ref[4]
        fine = np.isfinite(r)
        assert np.array_equal(g[~fine], r[~fine]) and np.all((np.abs(g - r) <= tol[:, None])[fine])


# rows, vocabulary, row length, likeliest, temperature
SIZES = [(1, 128256, 128256, 20, 1.0), (3, 128256, 128256, 64, 0.7), (2, 50257, 50264, 5, 1.0), (1, 1, 8, 1, 1.0), (5, 7, 8, 7, 2.0), (4, 64, 64, 64, 1.0),
         (2, 8193, 8200, 33, 1.0), (700, 4099, 4104, 3, 1.3), (2000, 513, 576, 1, 1.0), (1500, 1000, 1000, 64, 1.0), (40, 32000, 32000, 0, 0.9), (1100, 300, 304, 0, 1.0)]


@pytest.mark.parametrize("T,V,ld,n_top,temperature", SIZES)
def test_against_the_oracle(K, T, V, ld, n_top, temperature):
    rng = np.random.default_rng(T + V)
    b = si.f32_to_bf16_bits((rng.standard_normal((T, ld)) * 2.5).astype(np.float32))
    logits = dev_bf16(b)
    logits[:, V:] = float("nan")                          # behind the vocabulary: anything
    targets = rng.integers(0, V, T)
    if T > 2:
        targets[[0, T // 2]] = -100, V                    # not scored
        logits[0] = float("nan")
    z = si.bf16_bits_to_f64(b)[:, :V]
    t = torch.from_numpy(targets).cuda()
    got = forward(K, logits, t, V, 1 / temperature, n_top)
    check(got, z, targets, 1 / temperature, n_top)
    again = forward(K, logits, t, V, 1 / temperature, n_top)
    for x, y in zip(got, again):
        assert x is None or torch.equal(x, y)


def test_without_targets_and_with_outputs_left_out(K):
    rng = np.random.default_rng(0)
    b = si.f32_to_bf16_bits((rng.standard_normal((9, 3000)) * 2).astype(np.float32))
    z, logits = si.bf16_bits_to_f64(b), dev_bf16(b)
    check(forward(K, logits, None, 3000, 1.0, 4), z, None, 1.0, 4)
    full = forward(K, logits, torch.zeros(9, dtype=torch.int64, device="cuda"), 3000, 1.0, 4)
    for keep in range(5):
        out = [torch.empty_like(x) if i == keep else None for i, x in enumerate(full)]
        K.token_logprobs_forward(logits, torch.zeros(9, dtype=torch.int64, device="cuda"), 9, 3000, 3000, 1.0, 4, *out,
                                 workspace(K.token_logprobs_workspace_bytes(9, 3000, 4)))
        assert torch.equal(out[keep], full[keep])


def rows_of_every_kind(V, rng):
    x = rng.standard_normal((16, V)) * 3
    x[0] = 1.5                                            # all equal
    x[1] = np.arange(V) / V * 20 - 10                     # ascending: every vector holds new likeliest
    x[2] = -x[1]
    x[3] = -np.inf                                        # nothing left by the mask
    x[4] = -np.inf
    x[4, V - 1] = 2.0                                     # one left
    x[5, : V // 2] = -np.inf
    x[6] = np.where(np.arange(V) % 97 == 0, 0.0, -0.0)    # zeros of both signs are equal
    x[7] = np.float32(-3.3895313892515355e38)             # the type's lowest value
    x[8, 5] = np.float32(-3.3895313892515355e38)
    x[9] = -30.0
    x[9, 3] = 60.0                                        # all but certain
    x[10] = np.round(x[10])                               # many ties
    x[11] = 1000.0 + x[11]
    x[12] = x[12] * 100
    x[13, :] = -np.inf
    x[13, [2, V // 3, V - 2]] = [1.0, 1.0, -4.0]
    x[14] = np.sort(x[14])
    return si.f32_to_bf16_bits(x.astype(np.float32))


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("V", [40, 517, 2048, 33000])
def test_rows_of_every_kind(K, V, many):
    rng = np.random.default_rng(V)
    b = rows_of_every_kind(V, rng)
    if many:                                              # whole rows to a workgroup
        b = np.tile(b, (80, 1))
    n_top = 33
    ld = -(-V // 8) * 8
    padded = np.full((len(b), ld), 0x7F80, np.uint16)     # +infinity behind the vocabulary
    padded[:, :V] = b
    targets = rng.integers(0, V, len(b))
    targets[3::16], targets[4::16], targets[9::16] = 0, V - 1, 3
    got = forward(K, dev_bf16(padded), torch.from_numpy(targets).cuda(), V, 1.0, n_top)
    check(got, si.bf16_bits_to_f64(b), targets, 1.0, n_top)


def test_rows_that_are_not_finite(K):
    rng = np.random.default_rng(1)
    V, n_top = 9000, 4
    x = rng.standard_normal((4, V)).astype(np.float32)
    x[0, 4000] = np.nan
    x[1, 77] = np.inf
    x[2] = np.nan
    x[2, [8, 3]] = 1.0, 2.0
    got = forward(K, dev_bf16(si.f32_to_bf16_bits(x)), torch.tensor([5, 5, 5, 5], device="cuda"), V, 1.0, n_top)
    for g in (got[0], got[1], got[2], got[4]):
        g = g.cpu()
        assert g[:3].isnan().all() and g[3].isfinite().all()
    ids = got[3].cpu().numpy()
    assert ids[2].tolist() == [3, 8, -1, -1] and ids[1, 0] == 77 and (ids[0] >= 0).all()


@pytest.mark.parametrize("T,V,ld,temperature", [(3, 128256, 128256, 1.0), (70, 50257, 50304, 0.7), (1, 1, 8, 1.0), (500, 513, 576, 1.3), (2, 8200, 8200, 1.0)])
@pytest.mark.parametrize("which", ["both", "logprobs", "entropy"])
def test_gradient_against_the_oracle(K, T, V, ld, temperature, which):
    rng = np.random.default_rng(T + V)
    b = si.f32_to_bf16_bits((rng.standard_normal((T, ld)) * 2.5).astype(np.float32))
    z, logits = si.bf16_bits_to_f64(b)[:, :V], dev_bf16(b)
    logits[:, V:] = float("nan")
    targets = rng.integers(0, V, T)
    if T > 2:
        targets[1] = -1
        logits[1] = float("nan")
    t = torch.from_numpy(targets).cuda()
    dl = rng.standard_normal(T).astype(np.float32) if which != "entropy" else None
    dh = rng.standard_normal(T).astype(np.float32) if which != "logprobs" else None
    inverse = 1 / temperature
    _, h, lse, *_ = forward(K, logits, t, V, inverse)
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    ref = og.logprobs_gradient(z, targets, inverse, dl, dh)
    d = garbage((T, ld))
    K.token_logprobs_backward(logits, t, lse, h if dh is not None else None, dev(dl), dev(dh), T, V, ld, inverse, d)
    got = host_f64(d)
    assert np.all(got[:, V:] == 0)
    r = og.logprobs(z, targets, inverse, 0)
    size = np.abs(z) * inverse + np.abs(r[2])[:, None]
    p = np.exp(z * inverse - r[2][:, None]) * (r[2] != 0)[:, None]
    terms = p * (np.abs(dl)[:, None] if dl is not None else 0) + p * (np.abs(dh)[:, None] * (np.abs(z * inverse - r[2][:, None]) + r[1][:, None]) if dh is not None else 0)
    if dl is not None:
        for i in range(T):
            if 0 <= targets[i] < V:
                terms[i, targets[i]] += abs(dl[i])
    bound = 2.0 ** -8 * np.abs(ref) + 4e-6 * (1 + size) * terms * inverse + 1e-37
    assert np.all(np.abs(got[:, :V] - ref) <= 1.001 * bound), np.max(np.abs(got[:, :V] - ref) / bound)
    # in place
    K.token_logprobs_backward(logits, t, lse, h, dev(dl), dev(dh), T, V, ld, inverse, logits)
    assert torch.equal(logits.view(torch.int16), d.view(torch.int16))


def test_gradient_of_rows_of_every_kind(K):
    rng = np.random.default_rng(3)
    V = 2048
    b = rows_of_every_kind(V, rng)
    z, logits = si.bf16_bits_to_f64(b), dev_bf16(b)
    targets = rng.integers(0, V, len(b))
    targets[4], targets[9] = V - 1, 3
    t = torch.from_numpy(targets).cuda()
    dl, dh = rng.standard_normal(len(b)), rng.standard_normal(len(b))
    _, h, lse, *_ = forward(K, logits, t, V)
    d = garbage(b.shape)
    K.token_logprobs_backward(logits, t, lse, h, torch.from_numpy(dl).float().cuda(), torch.from_numpy(dh).float().cuda(), len(b), V, V, 1.0, d)
    ref = og.logprobs_gradient(z, targets, 1.0, dl, dh)
    got = host_f64(d)
    assert np.all(np.isfinite(got)) and np.all(got[3] == 0)
    size = np.where(np.isfinite(z), np.abs(z), 0.0).max(-1)[:, None]
    assert np.all(got[7] == 0)
    # p is off by 2^-24 of |z| + |lse|, which for a likely token is about the row's largest
    keep = size[:, 0] < 1e5
    assert keep.sum() == 14 and np.all(np.abs(got - ref)[keep] <= (2.0 ** -8 * np.abs(ref) + 1e-5 * (1 + size))[keep])


def test_gradient_against_differences(K):
    """The gradient of a sum of log-probabilities and entropies against differences of the oracle's forward along random directions."""
    rng = np.random.default_rng(8)
    T, V, inverse = 6, 700, 1.4
    b = si.f32_to_bf16_bits((rng.standard_normal((T, 704)) * 2).astype(np.float32))
    z, logits = si.bf16_bits_to_f64(b)[:, :V], dev_bf16(b)
    targets = rng.integers(0, V, T)
    dl, dh = rng.standard_normal(T), rng.standard_normal(T)
    t = torch.from_numpy(targets).cuda()
    _, h, lse, *_ = forward(K, logits, t, V, inverse)
    d = garbage((T, 704))
    K.token_logprobs_backward(logits, t, lse, h, torch.from_numpy(dl).float().cuda(), torch.from_numpy(dh).float().cuda(), T, V, 704, inverse, d)
    got = host_f64(d)[:, :V]

    def loss(x):
        r = og.logprobs(x, targets, inverse, 0)
        return float(np.sum(dl * r[0] + dh * r[1]))

    for _ in range(4):
        u = rng.standard_normal((T, V))
        eps = 1e-4
        slope = (loss(z + eps * u) - loss(z - eps * u)) / (2 * eps)
        # roundings of independent elements: 2^-8 of each at most, added up with random signs over at least 700 elements (6 deviations of 2^-8 / sqrt(3))
        assert abs(np.sum(got * u) - slope) <= 6 * 2.0 ** -8 / 3 ** 0.5 * np.sqrt(np.sum((got * u) ** 2)) + 1e-6 * abs(slope) + 1e-6


def test_captured_and_replayed_and_other_streams(K):
    rng = np.random.default_rng(6)
    for T, V in ((1, 20000), (2000, 800)):
        logits = torch.empty((T, V), dtype=torch.bfloat16, device="cuda")
        t = torch.zeros(T, dtype=torch.int64, device="cuda")
        out = [garbage((T,), torch.float32) for _ in range(3)] + [torch.zeros((T, 5), dtype=torch.int64, device="cuda"), garbage((T, 5), torch.float32)]
        ws, d, one = workspace(K.token_logprobs_workspace_bytes(T, V, 5)), garbage((T, V)), torch.ones(T, device="cuda")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            K.token_logprobs_forward(logits, t, T, V, V, 1.0, 5, *out, ws)
            K.token_logprobs_backward(logits, t, out[2], out[1], one, one, T, V, V, 1.0, d)
        for turn in range(4):
            logits.copy_(torch.randn((T, V), device="cuda") * 2)
            t.copy_(torch.randint(-1, V, (T,), device="cuda"))
            g.replay()
            torch.cuda.synchronize()
            want = forward(K, logits, t, V, 1.0, 5)
            grad = garbage((T, V))
            K.token_logprobs_backward(logits, t, want[2], want[1], one, one, T, V, V, 1.0, grad)
            for x, y in zip(out + [d], want + [grad]):
                assert torch.equal(x, y)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        other = forward(K, logits, t, V, 1.0, 5, side)
        side.synchronize()
        for x, y in zip(other, out):
            assert torch.equal(x, y)


def test_logits_of_more_than_4_gib(K):
    T, V = 17000, 128256
    logits = torch.full((T, V), -1.0, dtype=torch.bfloat16, device="cuda")
    targets = torch.randint(0, V, (T,), device="cuda")
    logits.scatter_(1, targets[:, None], 6.0)
    out = forward(K, logits, targets, V, 1.0, 2)
    s = np.exp(7.0) + V - 1
    assert torch.allclose(out[0], torch.full((T,), float(7.0 - np.log(s)), device="cuda"), atol=1e-5, rtol=0)
    assert torch.equal(out[3][:, 0], targets) and torch.equal(out[3][:, 1], (targets == 0).long())
    one = torch.ones(T, device="cuda")
    K.token_logprobs_backward(logits, targets, out[2], None, one, None, T, V, V, 1.0, logits)
    p = np.exp(7.0) / s
    got = logits.gather(1, targets[:, None]).float()
    assert torch.allclose(got, torch.full_like(got, float(1 - p)), rtol=2.0 ** -8, atol=0)
    assert torch.equal(logits[-1].float().max(), got[-1, 0])


def test_nothing_is_written_around_the_outputs(K):
    guard = 1024
    for T, V, ld, n in ((3, 20001, 20008, 7), (1200, 500, 504, 3)):
        logits = torch.randn((T, ld), device="cuda").bfloat16()
        t = torch.randint(0, V, (T,), device="cuda")
        sizes = [T, T, T, T * n, T * n]
        out = [torch.full((m + 2 * guard,), 7, dtype=torch.int64 if i == 3 else torch.float32, device="cuda") for i, m in enumerate(sizes)]
        nbytes = K.token_logprobs_workspace_bytes(T, V, n)
        ws = torch.full((nbytes + 2 * guard,), 77, dtype=torch.uint8, device="cuda")
        K.token_logprobs_forward(logits, t, T, V, ld, 1.0, n, *(x[guard:] for x in out), ws[guard:])
        d = torch.full((T * ld + 2 * guard,), 7.0, dtype=torch.bfloat16, device="cuda")
        K.token_logprobs_backward(logits, t, out[2][guard:], None, torch.ones(T, device="cuda"), None, T, V, ld, 1.0, d[guard:])
        for x, m in zip(out + [d], sizes + [T * ld]):
            assert (x[:guard] == 7).all() and (x[guard + m:] == 7).all()
        assert (ws[:guard] == 77).all() and (ws[guard + nbytes:] == 77).all()


@pytest.mark.parametrize("T,V,n_top", [(1, 33000, 20), (1, 3000, 5), (1100, 20000, 5)])
def test_nan_of_every_kind_hide_no_token(K, T, V, n_top):
    """Quiet and signalling NaN of both signs among the logits, one of them beside the likeliest: the row's sums are NaN, its likeliest those of the rest."""
    rng = np.random.default_rng(V)
    b = si.f32_to_bf16_bits((rng.standard_normal((T, V)) * 2.5).astype(np.float32))
    z, best = si.bf16_bits_to_f64(b), int(np.argmax(si.bf16_bits_to_f64(b)[0]))
    where = [best ^ 1, 17, V // 2 | 1, V - 1]
    where = [w if w != best else w - 2 for w in where]
    b[0, where] = 0x7F81, 0xFF81, 0x7FC0, 0xFFFF
    got = forward(K, dev_bf16(b), torch.full((T,), best, device="cuda"), V, 1.0, n_top)
    assert all(x[0].isnan() for x in got[:3]) and got[4][0].isnan().all()
    z[0, where] = -np.inf
    assert np.array_equal(got[3][0].cpu().numpy(), np.argsort(-z[0], kind="stable")[:n_top])
    if T > 1:
        assert all(x[1:].isfinite().all() for x in got[:3])


@pytest.mark.parametrize("V", [40, 517, 2048, 33000])
@pytest.mark.parametrize("which", ["both", "logprobs", "entropy"])
def test_gradient_of_rows_of_every_kind_element_by_element(K, V, which):
    """The bound of the gradient in its terms' magnitudes, which are those of p: the tails of a row are held to theirs, and not to the row's largest."""
    rng = np.random.default_rng(V)
    ld = -(-V // 8) * 8
    padded = np.full((16, ld), 0x7F80, np.uint16)         # +infinity behind the vocabulary
    padded[:, :V] = b = rows_of_every_kind(V, rng)
    z, logits = si.bf16_bits_to_f64(b), dev_bf16(padded)
    targets = rng.integers(0, V, 16)
    targets[4], targets[9], targets[12] = V - 1, 3, int(np.argmin(z[12]))
    t = torch.from_numpy(targets).cuda()
    dl = rng.standard_normal(16).astype(np.float32) if which != "entropy" else None
    dh = rng.standard_normal(16).astype(np.float32) if which != "logprobs" else None
    _, h, lse, *_ = forward(K, logits, t, V)
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    d = garbage((16, ld))
    K.token_logprobs_backward(logits, t, lse, h if dh is not None else None, dev(dl), dev(dh), 16, V, ld, 1.0, d)
    got = host_f64(d)
    assert np.all(got[:, V:] == 0)
    got = got[:, :V]
    ref = og.logprobs_gradient(z, targets, 1.0, dl, dh)
    r = og.logprobs(z, targets, 1.0, 0)
    left = ~(r[2] <= -1e30)                               # rows of which the mask has left something
    assert left.sum() == 14 and np.all(got[~left] == 0)
    got, ref, z, at = got[left], ref[left], z[left], targets[left]
    lse64, entropy = r[2][left][:, None], r[1][left][:, None]
    p = np.exp(z - lse64)
    logp = np.where(p > 0, z - lse64, 0.0)
    size = np.where(p > 0, np.abs(z), 0.0) + np.abs(lse64)
    terms = np.zeros_like(p)
    if dl is not None:
        terms += p * np.abs(dl[left])[:, None]
        terms[np.arange(len(at)), at] += np.abs(dl[left])
    if dh is not None:
        terms += p * np.abs(dh[left])[:, None] * (np.abs(logp) + entropy)
    # 1e-37: what fp32's exponential leaves of p below its smallest normal number, 2^-126.  The entropy is without the p |log p| of such tokens, each at most
    # 2^-126 * 126 ln 2 (p |log p| falls with p), of which a row has up to V: in the row that is all but certain they are all of it (2.4e-33 of V 33000)
    lost = V * 2.0 ** -126 * 126 * np.log(2) * p * (np.abs(dh[left])[:, None] if dh is not None else 0)
    bound = 2.0 ** -8 * np.abs(ref) + 4e-6 * (1 + size) * terms + 1e-37 * (1 + size) + lost
    assert np.all(np.abs(got - ref) <= 1.001 * bound), np.max(np.abs(got - ref) / bound)
