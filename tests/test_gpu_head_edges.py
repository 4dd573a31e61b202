"""Log probabilities and cross entropy at the ends of their ranges, on the GPU against the oracle."""
import numpy as np
import pytest
import torch

import paper_2107_13490_amd as pkg
from gpu_util import ctx, dev, host
from oracle import fxp_oracle as orc
from oracle import head_oracle as head
from test_gpu_head import EPS, _fl, _logits, _near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,classes", [(4000, 250), (4000, 300), (200, 6007), (4, 300007)])
@pytest.mark.parametrize("wl_g", [8, 16, 24])
def test_masked_classes_have_no_gradient_whatever_the_weight(rows, classes, wl_g):
    """A class of p = 0 has a gradient of 0 and not of "a little below 0", which a draw of 0 would round to -1."""
    rng = np.random.default_rng([rows, classes])
    x = rng.normal(size=(rows, classes)).astype(np.float32)
    y, w = rng.integers(0, classes, rows), -0.5 - rng.random(rows).astype(np.float32)
    masked = rng.random((rows, classes)) < 0.5
    masked[np.arange(rows), y] = False
    low = masked & (rng.random((rows, classes)) < 0.5)
    x[masked], x[low] = -np.inf, np.finfo(np.float32).min
    zero = orc.rounding_bits(x.size, orc.SR, 3, 5).reshape(x.shape) == 0
    assert (zero & masked & ~low).any() and (zero & low).any() and (zero & ~masked).any()
    got = host(ctx().cross_entropy(dev(x), None, dev(y), (wl_g, wl_g - 1), weights=dev(w), seed=3, stream=5)[0])
    assert not got[masked].any()
    assert np.array_equal(got, head.quantize_real(head.gradient(x, None, y, w), wl_g, wl_g - 1, seed=3, stream=5))


@pytest.mark.parametrize("at", [1e10, -1e10, 2.0 ** 33, -2.0 ** 33, 2.0 ** 34 - 4096, 2.0 ** 32, -3e9, 1e12])
@pytest.mark.parametrize("rows,classes", [(3, 200), (3, 20000), (3, 60000)])
def test_large_logits_one_step_apart(at, rows, classes):
    """Logits whose neighbours in fp32 are 256 to 65536 apart: the larger ones share the row."""
    x = np.full((rows, classes), at, dtype=np.float32)
    up = np.nextafter(np.float32(at), np.float32(np.inf))
    x[0, classes // 2::classes // 8] = up
    x[1, -1] = up
    y = np.array([classes // 2, classes - 1, 3])
    got, logp = ctx().cross_entropy(dev(x), None, dev(y), (16, 15), seed=3, stream=5)
    want = head.log_probs(x, None, y, 3)
    _near(host(logp), want["logp"], EPS * np.abs(want["logp"]) + 2.0 ** -40, "logp")
    assert np.array_equal(host(got), head.quantize_real(head.gradient(x, None, y), 16, 15, seed=3, stream=5))
    assert np.array_equal(host(ctx().log_probs(dev(x), None, dev(y), topk=3)["top_idx"]), want["top_idx"])


@pytest.mark.parametrize("rows,classes", [(127, 10), (127, 300), (127, 5000), (60, 200003)])
@pytest.mark.parametrize("f", [(8, 3), (8, 4), (8, 1), (12, 7), (16, 8), (24, 18), None])
def test_probabilities_are_at_most_one(rows, classes, f):
    """Rows with one class that has nearly all of it: its log probability is rounded to 0 at most."""
    c = np.arange(1, rows + 1)
    y = (c * 7919) % classes
    if f is None:
        x = np.full((rows, classes), -40, dtype=np.float32)
        x[np.arange(rows), y] = c / 8 + 0.1
    else:
        x = np.full((rows, classes), -(1 << (f[0] - 1)), dtype=np.int8 if f[0] <= 8 else np.int16 if f[0] <= 16 else np.int32)
        x[np.arange(rows), y] = c * 2 ** (f[0] - 8)
    r = ctx().log_probs(dev(x), f, dev(y), topk=2)
    logp = host(ctx().cross_entropy(dev(x), f, dev(y), (8, 7))[1])
    for v in (host(r["logp"]), host(r["top_logp"]), logp):
        assert v.max() <= 0, v.max()
    assert np.array_equal(host(r["top_idx"])[:, 0], y)


@pytest.mark.parametrize("rows,classes", [(9, 3), (9, 200), (9, 3000), (9, 70001)])
def test_a_certain_class_has_the_logarithm_of_one(rows, classes):
    x = np.full((rows, classes), -np.inf, dtype=np.float32)
    y = (np.arange(rows) * 31) % classes
    x[np.arange(rows), y] = np.linspace(-700, 700, rows)
    assert not host(ctx().cross_entropy(dev(x), None, dev(y), (8, 7))[1]).any()
    r = ctx().log_probs(dev(x), None, dev(y), topk=1)
    assert not host(r["logp"]).any() and not host(r["top_logp"]).any() and not host(r["entropy"]).any()
    assert np.array_equal(host(r["lse"]), x[np.arange(rows), y])


@pytest.mark.parametrize("rows,classes", [(40, 100), (40, 2000), (200, 5001), (3, 60001)])
@pytest.mark.parametrize("wl", [0, 8, 12, 16, 24])
def test_the_loss_has_all_of_its_bits(rows, classes, wl):
    """Sum and logarithm are in 64 bits: beside the rounding of the result there are only theirs, at most 2^11 additions
    in a row (2^-42), exponentials and logarithm (2^-48 together)."""
    rng = np.random.default_rng([rows, classes, wl])
    x = _logits(rng, rows, classes, wl, _fl(wl))
    y = rng.integers(0, classes, rows)
    if wl == 0:
        x[np.arange(rows), y] = rng.random(rows) * 30
    else:
        lim = (1 << (wl - 1)) - 1
        x[np.arange(rows), y] = np.rint(lim * rng.random(rows)).astype(x.dtype)
    logp = ctx().cross_entropy(dev(x), (wl, _fl(wl)) if wl else None, dev(y), (8, 7))[1]
    want = head.log_probs(x, _fl(wl) if wl else None, y, 0)["logp"]
    _near(host(logp), want, EPS * np.abs(want) + 2.0 ** -41, "logp")


def test_gradients_beside_the_logits_but_not_in_their_place():
    rng = np.random.default_rng(2)
    x, y = _logits(rng, 6, 300, 8, 4), rng.integers(0, 300, 6)
    both = torch.zeros((6, 640), dtype=torch.int8, device="cuda")
    both[:, 20:320] = dev(x)
    t = both[:, 20:320]
    for out in (t, both[:, 21:321], both[:, :300], both[:, 319:619]):
        with pytest.raises(pkg.AdaptError):
            ctx().cross_entropy(t, (8, 4), dev(y), (8, 7), out=out)
    assert np.array_equal(host(t), x)
    ctx().cross_entropy(t, (8, 4), dev(y), (8, 7), seed=1, stream=2, out=both[:, 320:620])
    both = host(both)
    assert np.array_equal(both[:, 20:320], x) and not both[:, :20].any() and not both[:, 620:].any()
    assert np.array_equal(both[:, 320:620], head.quantize_real(head.gradient(x, 4, y), 8, 7, seed=1, stream=2))
