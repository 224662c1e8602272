"""The paged cache, the attention over it and the log-probabilities together, as examples/paged_generation.py runs them: a layer's weights on tokens that come a few at a
time, against the fp64 oracle of the whole row; and generation against the training step's forward.

Tolerances.  The layer's own (2e-2 of an element, cosine 0.999): the same roundings lie behind an output, and the weights of the attention are rounded as
there.  With an e4m3 cache the attention is held to the cache's own content, read back from it (the tolerances of the attention's test).  A logit has a rounding to bf16 in each of
some ten operands for a layer, 1.7e-3 rms of a logit's deviation s each: between two ways to the same logit, over L layers, 2 * sqrt(10 L) * 1.7e-3 * s rms, of which
six are allowed for the largest of some hundreds; a log-probability is a logit less a mean of logits.
"""
import numpy as np
import pytest
import torch

from oracle import decoder_layer as odl
from oracle import generation as og
from oracle import lm_stack as olm
from synth import inputs as si
from tests.parity import assert_close, host_f64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def E():
    from examples import paged_generation
    return paged_generation


CFG = si.LayerConfig(3, 128, 256, 8, 2, 64, 384, 1e-5, 10000.0)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_a_layer_on_tokens_a_few_at_a_time(E, e4m3, layout):
    cfg = CFG.with_(rope_layout=layout)
    model = E.Model(cfg, 1, 512, seed=3)
    g = E.Generator(model, 3, 128, e4m3)
    ids = torch.randint(512, (3, 128), generator=torch.Generator().manual_seed(5)).cuda()
    w = {n: host_f64(t) for n, t in model.layers[0].items()}
    x = olm.embed_fwd(host_f64(model.embed), ids.cpu().numpy().reshape(-1)).reshape(3, 128, -1)
    f = odl.layer_forward(cfg, x, w)
    at, got = [0, 0, 0], np.zeros(f["y"].shape)
    for counts in ([70, 0, 33], [1, 1, 1], [50, 64, 17], [1, 0, 1], [6, 63, 5], [0, 0, 64], [0, 0, 7]):
        S = max(counts)
        some = torch.zeros((3, S), dtype=torch.int64, device="cuda")
        for b, n in enumerate(counts):
            some[b, :n] = ids[b, at[b]:at[b] + n]
        y = host_f64(g.extend(some, counts)).reshape(3, S, -1)
        for b, n in enumerate(counts):
            got[b, at[b]:at[b] + n] = y[b, :n]
            at[b] += n
    assert at == [128, 128, 128] and g.tokens.tolist() == at and not g.free
    k, v = (torch.empty((3, 128, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    E.K.kv_cache_read(g.caches[0], None, None, 128, k, v)
    if not e4m3:
        assert_close(k, f["k"], "keys")
        assert_close(v, f["v"], "values")
        assert_close(got, f["y"], "layer output")
        return
    # keys and values: a rounding to e4m3 (half of 2^-3 of a binade, of 2^-9 units of the vector's power of two below) on top of the layer's own to bf16
    for held, ref in ((host_f64(k), f["k"]), (host_f64(v), f["v"])):
        unit = np.abs(ref).max(-1, keepdims=True) / 224
        assert np.all(np.abs(held - ref) <= 2.0 ** -4 * 1.05 * np.abs(ref) + 2.0 ** -9 * unit + 2e-2 * np.abs(ref).std())
    # the layer's output with the attention over what the cache holds
    q = f["q"]
    cache = {"k": host_f64(k).transpose(0, 2, 1, 3), "v": host_f64(v).transpose(0, 2, 1, 3), "page_table": np.arange(3)[:, None]}
    o, *_ = og.attention(cache, q, None, None, 64 ** -0.5)
    y1 = x + o.reshape(3, 128, -1) @ w["wo"].T
    h2, _ = odl.rmsnorm_fwd(y1, w["g_mlp"], cfg.rms_eps)
    assert_close(got, y1 + odl.swiglu_fwd(h2 @ w["w_gate"].T, h2 @ w["w_up"].T) @ w["w_down"].T, "layer output over the e4m3 cache")


@pytest.mark.parametrize("piece", [16, 200])
def test_generation_against_the_training_steps_forward(E, piece):
    cfg, n = CFG.with_(batch=3), 20
    model = E.Model(cfg, 2, 1024, seed=7)
    lengths = [1, 61, 100]
    ids = torch.randint(1024, (3, 100), generator=torch.Generator().manual_seed(2)).cuda()
    g = E.Generator(model, 3, 128)
    tokens, logp, entropy = g.generate(g.prompt(ids, lengths, piece), n)
    rows, targets = torch.zeros((3, 128), dtype=torch.int64, device="cuda"), torch.full((3, 128), -1, dtype=torch.int64, device="cuda")
    for b, m in enumerate(lengths):
        rows[b, :m], rows[b, m:m + n], targets[b, m - 1:m - 1 + n] = ids[b, :m], tokens[b], tokens[b]
    logits = model.whole_rows(rows)
    again = E.scores(logits, targets.view(-1)).view(3, 128)
    again = torch.stack([again[b, m - 1:m - 1 + n] for b, m in enumerate(lengths)])
    bound = 6 * 2 * (10 * 2) ** 0.5 * 1.7e-3 * float(logits.float().std())
    assert float((again - logp).abs().max()) <= bound
    # what was taken is the likeliest of the whole rows' logits too, up to that
    best = torch.log_softmax(logits.float(), -1).amax(-1).view(3, 128)
    best = torch.stack([best[b, m - 1:m - 1 + n] for b, m in enumerate(lengths)])
    assert float((best - again).max()) <= 2 * bound
    assert bool((entropy > 0).all()) and bool((entropy <= np.log(1024)).all())


def test_the_example_runs(E, capsys):
    E.main(n_layers=1, n=4)
    out = capsys.readouterr().out
    assert "bf16 cache: 16 tokens" in out and "e4m3 cache: 16 tokens" in out
