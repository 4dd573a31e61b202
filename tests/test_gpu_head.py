"""Log probabilities and cross entropy on the GPU against the oracle: gradient codes and the indices of the largest logits
equal, floating outputs within bounds that follow from their arithmetic.

Bound of the fp32 outputs, with eps = 2^-24 (half a step): a sum of exponentials is made of chains of at most 128 fp32
additions (fp64 from there on), of terms whose exponential is good to 2 eps + |x - ref| eps, |x - ref| <= 16 where the
reference is not the row's maximum and weighted with exp(-|x - ref|) <= 1/e where it is: relative error A = (128 + 2 + 16) eps.
That is an absolute error of the log of the sum, to which the rounding of the result adds eps |result|; of a log probability
the reference's rounding adds eps |ref|.  The entropy's second sum has the error A relative to sum p |x - ref|.
"""
import numpy as np
import pytest
import torch

import paper_2107_13490_amd as pkg
from gpu_util import ctx, dev, host
from oracle import fxp_oracle as orc
from oracle import head_oracle as head

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
A = (128 + 2 + 16) * EPS


def _np(wl):
    return np.float32 if wl == 0 else np.int8 if wl <= 8 else np.int16 if wl <= 16 else np.int32


def _logits(rng, rows, classes, wl, fl, spread=2.0):
    x = rng.normal(size=(rows, classes)) * spread
    if wl == 0:
        return x.astype(np.float32)
    lim = 1 << (wl - 1)
    return np.clip(np.rint(x * 2.0 ** fl), -lim, lim - 1).astype(_np(wl))


def _fl(wl):
    return max(0, wl - 5)


def _near(got, want, bound, what):
    got, want = np.asarray(got, dtype=np.longdouble), np.asarray(want, dtype=np.longdouble)
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)]), what
    off = np.abs(got - want)[fin] - np.broadcast_to(bound, want.shape)[fin]
    assert off.size == 0 or off.max() <= 0, (what, float(off.max()))


def _check_log_probs(x, f, labels, topk, t=None):
    fl = f[1] if f else None
    got = ctx().log_probs(dev(x) if t is None else t, f, None if labels is None else dev(labels), topk=topk)
    got = {k: host(v) for k, v in got.items() if v is not None}
    want = head.log_probs(x, fl, labels, topk)
    size = A + EPS * (np.abs(want["lse"].astype(float)) + np.where(np.isfinite(want["scale"]), want["scale"], 0).astype(float))
    size = np.where(np.isfinite(size), size, 0)
    _near(got["lse"], want["lse"], size, "lse")
    if labels is not None:
        _near(got["logp"], want["logp"], size + EPS * np.abs(want["logp"]), "logp")
    _near(got["entropy"], want["entropy"], A * (1 + want["scale"]) + 2 * size, "entropy")
    if topk:
        assert np.array_equal(got["top_idx"], want["top_idx"])
        _near(got["top_logp"], want["top_logp"], size[:, None] + EPS * np.abs(want["top_logp"]), "top_logp")


def _check_cross_entropy(x, f, labels, fg, weights=None, mode=pkg.SR, t=None, seed=3, stream=5):
    fl = f[1] if f else None
    got, logp = ctx().cross_entropy(dev(x) if t is None else t, f, dev(labels), fg, weights=None if weights is None else dev(weights),
                                    mode=mode, seed=seed, stream=stream)
    want = head.quantize_real(head.gradient(x, fl, labels, weights), *fg, mode=mode, seed=seed, stream=stream)
    got = host(got)
    assert got.dtype == _np(fg[0]) and np.array_equal(got, want), (np.argwhere(got != want)[:4], (got != want).sum())
    w = head.log_probs(x, fl, labels, 0)
    size = A + EPS * (np.abs(w["lse"].astype(float)) + w["scale"].astype(float) + np.abs(w["logp"].astype(float)))
    _near(host(logp), w["logp"], np.where(np.isfinite(size), size, 0), "logp")


def _labels(rng, rows, classes, ignored=0.2):
    y = rng.integers(0, classes, rows)
    y[rng.random(rows) < ignored] = -1
    return y.astype(np.int64)


SIZES = [(1, 1), (3, 2), (5, 7), (4, 8), (9, 9), (128, 10), (256, 100), (33, 129), (7, 1000), (5, 4099), (3, 8191), (2, 32768), (1, 70001),
         (2, 140003), (1, 300007)]


@pytest.mark.parametrize("rows,classes", SIZES)
@pytest.mark.parametrize("wl", [0, 8, 12, 16, 24])
def test_log_probs_sizes(rows, classes, wl):
    rng = np.random.default_rng([rows, classes, wl])
    x = _logits(rng, rows, classes, wl, _fl(wl))
    _check_log_probs(x, (wl, _fl(wl)) if wl else None, _labels(rng, rows, classes), min(classes, 5))


@pytest.mark.parametrize("rows,classes", SIZES)
@pytest.mark.parametrize("wl,wl_g", [(0, 8), (0, 20), (8, 8), (8, 16), (12, 12), (16, 8), (16, 16), (24, 8), (24, 24)])
def test_cross_entropy_sizes(rows, classes, wl, wl_g):
    rng = np.random.default_rng([rows, classes, wl, wl_g])
    x = _logits(rng, rows, classes, wl, _fl(wl))
    _check_cross_entropy(x, (wl, _fl(wl)) if wl else None, _labels(rng, rows, classes), (wl_g, wl_g - 1))


@pytest.mark.parametrize("f", [(2, 0), (4, 0), (8, 0), (8, 7), (8, 31), (9, 0), (16, 0), (16, 5), (16, 6), (16, 15), (16, 31), (17, 0), (32, 0), (32, 31), (32, 20)])
def test_formats_of_logits(f):
    """Codes over the whole range: values from +-2^31 down to differences that no exponential sees."""
    rng = np.random.default_rng(f)
    lim = 1 << (f[0] - 1)
    x = rng.integers(-lim, lim, (6, 777)).astype(_np(f[0]))
    x[1] = x[1] // 2 ** max(0, f[0] - 6)                      # close together
    x[2] = lim - 1                                            # all equal, at the ends
    x[3] = -lim
    x[4, 1:] = -lim                                           # one far above the rest
    y = _labels(rng, 6, 777)
    _check_log_probs(x, f, y, 7)
    for fg in ((8, 7), (16, 15), (16, 20)):
        _check_cross_entropy(x, f, y, fg)


@pytest.mark.parametrize("fg", [(2, 1), (4, 0), (8, 12), (8, 31), (16, 0), (16, 31), (24, 23), (32, 16)])
@pytest.mark.parametrize("mode", [pkg.SR, pkg.RN_HALF_UP])
def test_formats_of_gradients(fg, mode):
    rng = np.random.default_rng(fg)
    x = _logits(rng, 40, 321, 12, 7, spread=4.0)
    w = rng.normal(size=40).astype(np.float32) * 3
    _check_cross_entropy(x, (12, 7), _labels(rng, 40, 321), fg, weights=w, mode=mode)


@pytest.mark.parametrize("wl", [0, 8, 16, 32])
@pytest.mark.parametrize("topk", [0, 1, 2, 16, 31, 32])
def test_many_alternatives(wl, topk):
    rng = np.random.default_rng([wl, topk])
    for rows, classes in ((5, 32), (3, 700), (2, 20000), (1, 100001)):
        x = _logits(rng, rows, classes, wl, _fl(wl))
        _check_log_probs(x, (wl, _fl(wl)) if wl else None, None, topk)


@pytest.mark.parametrize("classes", [33, 1000, 50000, 200000])
@pytest.mark.parametrize("wl", [0, 4, 8, 16])
def test_ties_go_to_the_lowest_index(classes, wl):
    rng = np.random.default_rng([classes, wl])
    f = (wl, 1) if wl else None
    x = np.zeros((6, classes), dtype=_np(wl))                 # all equal
    x[1, classes // 2:] = 3                                   # a block of equal ones in the second half
    x[2] = np.arange(classes) % 7                             # the largest spread out
    x[3] = np.sort(rng.integers(-5, 6, classes))              # ascending
    x[4] = np.sort(rng.integers(-5, 6, classes))[::-1]        # descending
    x[5, -17:] = np.arange(17) // 2 - 4                       # at the end
    if wl == 0:
        x[0, ::2] = -0.0
    _check_log_probs(x, f, None, 32)
    _check_log_probs(x, f, None, 3)


@pytest.mark.parametrize("classes", [64, 4096, 100000])
def test_large_logits_side_by_side(classes):
    """The largest logits in one place, and many more of them than are asked for: ascending and descending runs."""
    x = np.full((4, classes), -3.0, dtype=np.float32)
    n = min(classes // 2, 3000)
    x[0, :n] = np.arange(n) * 1e-3
    x[1, -n:] = np.arange(n) * 1e-3
    x[2, 10:10 + n] = -np.arange(n) * 1e-3
    x[3] = np.arange(classes) * 1e-4
    _check_log_probs(x, None, None, 32)


def test_masks_infinities_and_nan():
    rng = np.random.default_rng(2)
    for classes in (3, 100, 5000, 70000):
        x = rng.normal(size=(10, classes)).astype(np.float32)
        low = np.finfo(np.float32).min
        x[0] = -np.inf                                         # nothing left
        x[1, 1:] = -np.inf                                     # one left
        x[2, classes // 2] = np.nan
        x[3, -1] = np.inf
        x[4] = low                                             # masked with the type's lowest value, all of it
        x[5, : classes // 2] = low
        x[6, 0], x[6, 1] = -np.inf, 3e38
        x[7] = -np.inf
        x[7, -1] = low
        x[8, :] = np.nan
        x[9, ::2] = -np.inf
        y = np.array([0, 0, 1, 1, 2, 0, 1, classes - 1, 0, 1])
        with np.errstate(invalid="ignore"):
            _check_log_probs(x, None, y, 3)
            _check_cross_entropy(x, None, y, (16, 15))
            y[:] = [1, 2, -1, -1, -1, 1, 0, 0, -1, 0]
            _check_log_probs(x, None, y, 1)
            _check_cross_entropy(x, None, y, (8, 7))


def test_labels_out_of_range_and_none():
    rng = np.random.default_rng(6)
    x = _logits(rng, 5, 100, 8, 4)
    y = np.array([100, 1 << 40, -(1 << 40), 99, 0])
    _check_log_probs(x, (8, 4), y, 2)
    _check_cross_entropy(x, (8, 4), y, (8, 7))
    _check_cross_entropy(x, (8, 4), np.full(5, -1), (8, 7))


@pytest.mark.parametrize("wl", [0, 8, 16, 24])
@pytest.mark.parametrize("pad,lo", [(1, 0), (3, 1), (8, 2), (5, 5)])
def test_strided_rows_and_unaligned_bases(wl, pad, lo):
    rng = np.random.default_rng([wl, pad, lo])
    for rows, classes in ((6, 37), (5, 2051), (2, 40007)):
        whole = _logits(rng, rows, classes + pad + lo, wl, _fl(wl))
        x = np.ascontiguousarray(whole[:, lo:lo + classes])
        t = dev(whole)[:, lo:lo + classes]
        f = (wl, _fl(wl)) if wl else None
        y = _labels(rng, rows, classes)
        _check_log_probs(x, f, y, 4, t=t)
        _check_cross_entropy(x, f, y, (8, 7), t=t)
        wide = torch.full((rows, classes + 7), 55, dtype=torch.int16, device="cuda")
        out = wide[:, 3:3 + classes]
        got, _ = ctx().cross_entropy(t, f, dev(y), (16, 15), seed=1, stream=2, out=out)
        want = head.quantize_real(head.gradient(x, f[1] if f else None, y), 16, 15, seed=1, stream=2)
        wide = host(wide)
        assert np.array_equal(wide[:, 3:3 + classes], want)
        assert np.all(wide[:, :3] == 55) and np.all(wide[:, 3 + classes:] == 55)


def test_many_rows():
    rng = np.random.default_rng(11)
    for rows, classes, wl in ((5000, 10, 8), (3001, 65, 16), (700, 1500, 8), (70000, 3, 0)):
        x = _logits(rng, rows, classes, wl, _fl(wl))
        y = _labels(rng, rows, classes)
        f = (wl, _fl(wl)) if wl else None
        _check_log_probs(x, f, y, 2)
        _check_cross_entropy(x, f, y, (8, 7))


def test_weights_of_every_kind():
    rng = np.random.default_rng(8)
    w = np.array([0.0, -0.0, -1.5, 3e38, -3e38, np.inf, -np.inf, np.nan, 1e-40, 2.0], dtype=np.float32)
    finite = np.where(np.isfinite(w), w, 0).astype(np.float32)
    for rows, classes, wl in ((10, 90, 8), (10, 3001, 8), (10, 3001, 16), (10, 3001, 0), (10, 70001, 0)):
        x, y = _logits(rng, rows, classes, wl, _fl(wl)), rng.integers(0, classes, rows)
        f = (wl, _fl(wl)) if wl else None
        got, logp = ctx().cross_entropy(dev(x), f, dev(y), (12, 11), weights=dev(w), seed=3, stream=5)
        want = head.quantize_real(head.gradient(x, f[1] if f else None, y, finite), 12, 11, seed=3, stream=5)
        assert np.array_equal(host(got), want)
        assert np.isfinite(host(logp)).all()


@pytest.mark.parametrize("rows,classes", [((1 << 21) + 5, 300), ((1 << 23) + 9, 3)])
def test_more_rows_than_a_launch_takes(rows, classes):
    """Rows around the seam and at the end, against calls on those rows alone (nearest rounding: no draws)."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-60, 60, (rows, classes), generator=g, device="cuda", dtype=torch.int8)
    y = torch.randint(-1, classes, (rows,), generator=g, device="cuda")
    c = ctx()
    lp = c.log_probs(x, (8, 4), y, topk=2)
    dl, logp = c.cross_entropy(x, (8, 4), y, (8, 7), mode=pkg.RN_HALF_UP)
    seam = 1 << (21 if classes > 256 else 23)
    for a, b in ((0, 4), (seam - 3, seam + 3), (rows - 4, rows)):
        want = c.log_probs(x[a:b], (8, 4), y[a:b], topk=2)
        for k in want:
            assert torch.equal(lp[k][a:b], want[k]), (k, a)
        w, wp = c.cross_entropy(x[a:b].clone(), (8, 4), y[a:b], (8, 7), mode=pkg.RN_HALF_UP)
        assert torch.equal(dl[a:b], w) and torch.allclose(logp[a:b], wp, rtol=1e-6, atol=1e-6)
        assert torch.equal(logp[a:b] == 0, y[a:b] < 0)


def test_gradient_against_differences_of_the_loss():
    """(L(x + h) - L(x - h)) / 2h of the oracle's loss against the codes' values: half a code step for the rounding, h^2 / 6
    for the third derivative (below 1), and the difference's own rounding, 2^-63 |L| / h."""
    rng = np.random.default_rng(7)
    x, y, w = rng.normal(size=(6, 50)).astype(np.float32), _labels(rng, 6, 50), rng.random(6).astype(np.float32)
    got, logp = ctx().cross_entropy(dev(x), None, dev(y), (24, 22), weights=dev(w), mode=pkg.RN_HALF_UP)
    g, h = host(got) * 2.0 ** -22, np.longdouble(2.0 ** -12)
    assert abs(float(-(host(logp).astype(np.float64) * w).sum() - float(head.loss(x, None, y, w)))) <= 6 * 10 * A
    for i, j in [(i, j) for i in range(6) for j in (0, 1, int(max(y[i], 2)), 49)]:
        up, down = x.astype(np.longdouble), x.astype(np.longdouble)
        up[i, j] += h
        down[i, j] -= h
        d = (head.loss(up, None, y, w) - head.loss(down, None, y, w)) / (2 * h)
        assert abs(float(d) - g[i, j]) <= 2.0 ** -23 + float(h) ** 2 / 6 + 2.0 ** -63 * 40 / float(h)


def test_without_optional_outputs():
    rng = np.random.default_rng(1)
    x = dev(_logits(rng, 9, 200, 8, 4))
    r = ctx().log_probs(x, (8, 4), entropy=False)
    assert r["logp"] is None and r["entropy"] is None and r["top_idx"] is None
    assert torch.equal(r["lse"], ctx().log_probs(x, (8, 4), topk=3)["lse"])


def test_same_results_every_time_and_with_a_small_workspace():
    """The same call gives the same bits, whatever ran in the workspace before."""
    rng = np.random.default_rng(5)
    x, y = dev(_logits(rng, 3, 200003, 16, 11)), dev(_labels(rng, 3, 200003, 0))
    c = pkg.Context(workspace_bytes=1 << 20)
    first = [c.log_probs(x, (16, 11), y, topk=9), c.cross_entropy(x, (16, 11), y, (16, 15))]
    for k in range(4):
        c.quantize(torch.randn(100000, device="cuda"), 8, 4)
        again = [c.log_probs(x, (16, 11), y, topk=9), c.cross_entropy(x, (16, 11), y, (16, 15))]
        for name in first[0]:
            assert torch.equal(first[0][name], again[0][name])
        assert torch.equal(first[1][0], again[1][0]) and torch.equal(first[1][1], again[1][1])


def test_captured_and_replayed():
    rng = np.random.default_rng(3)
    shapes = [(64, 10, 8), (2, 150001, 8), (40, 9000, 16), (3, 80000, 0)]
    xs = [dev(_logits(rng, r, n, wl, _fl(wl))) for r, n, wl in shapes]
    ys = [dev(_labels(rng, r, n, 0.1)) for r, n, _ in shapes]
    fs = [(wl, _fl(wl)) if wl else None for _, _, wl in shapes]
    stream = torch.cuda.Stream()
    c = pkg.Context(stream=stream)
    stream.wait_stream(torch.cuda.current_stream())

    def calls(who):
        out = []
        for x, y, f in zip(xs, ys, fs):
            out += [v for v in who.log_probs(x, f, y, topk=6).values()]
            out += who.cross_entropy(x, f, y, (8, 7), seed=4, stream=9)
        return out

    with torch.cuda.stream(stream):
        calls(c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        outs = calls(c)
    for k in range(4):
        for x in xs:
            x.copy_(x.roll(k + 1, 1))
        want = calls(ctx())
        torch.cuda.synchronize()
        for v in outs:
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for v, w in zip(outs, want):
            assert torch.equal(v, w)


def test_empty_batches():
    x = torch.empty((0, 10), dtype=torch.int8, device="cuda")
    y = torch.empty(0, dtype=torch.int64, device="cuda")
    assert ctx().log_probs(x, (8, 4), y, topk=2)["top_idx"].shape == (0, 2)
    assert ctx().cross_entropy(x, (8, 4), y, (8, 7))[0].shape == (0, 10)


def test_offsets_past_32_bits():
    """A row that lies behind the first 2^32 bytes, of logits and of gradients."""
    rows, classes = 3, 65537
    ld = (1 << 31) + 8
    x = torch.zeros(2 * ld + classes, dtype=torch.int8, device="cuda")
    rng = np.random.default_rng(1)
    v = _logits(rng, rows, classes, 8, 4)
    t = torch.as_strided(x, (rows, classes), (ld, 1))
    t.copy_(dev(v))
    y = _labels(rng, rows, classes, 0)
    _check_log_probs(v, (8, 4), y, 5, t=t)
    out = torch.as_strided(torch.zeros(2 * ld + classes, dtype=torch.int8, device="cuda"), (rows, classes), (ld, 1))
    got, _ = ctx().cross_entropy(t, (8, 4), dev(y), (8, 7), seed=1, stream=2, out=out)
    assert np.array_equal(host(got.contiguous()), head.quantize_real(head.gradient(v, 4, y), 8, 7, seed=1, stream=2))


def test_refusals():
    c = ctx()
    x = torch.zeros((4, 20), dtype=torch.int8, device="cuda")
    y = torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (dict(topk=33), dict(topk=21), dict(topk=-1), dict(f=(8, 32)), dict(f=(1, 0))):
        with pytest.raises(pkg.AdaptError):
            c.log_probs(x, **{"f": (8, 4), "labels": y, **bad})
    for bad in (dict(fg=(33, 0)), dict(fg=(8, -1)), dict(mode=3), dict(f=(8, 40))):
        with pytest.raises(pkg.AdaptError):
            c.cross_entropy(x, **{"f": (8, 4), "labels": y, "fg": (8, 7), **bad})
    for call in (lambda: c.log_probs(x, None, y), lambda: c.log_probs(x, (16, 4), y), lambda: c.log_probs(x.t(), (8, 4), y),
                 lambda: c.log_probs(x[0], (8, 4), y), lambda: c.log_probs(x, (8, 4), y[:3]), lambda: c.log_probs(x, (8, 4), y.int()),
                 lambda: c.log_probs(x[:1].expand(4, 20), (8, 4), y), lambda: c.log_probs(x.cpu(), (8, 4), y),
                 lambda: c.cross_entropy(x, (8, 4), y, (8, 7), weights=torch.zeros(4, device="cuda", dtype=torch.float64)),
                 lambda: c.cross_entropy(x, (8, 4), y, (8, 7), out=torch.zeros((4, 20), dtype=torch.int16, device="cuda")),
                 lambda: c.cross_entropy(x, (8, 4), y.cpu(), (8, 7))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(pkg.AdaptError):
        c.log_probs(torch.zeros((4, 0), dtype=torch.int8, device="cuda"), (8, 4), y)


@pytest.mark.parametrize("wl", [0, 8, 16])
def test_fewer_chunks_than_alternatives(wl):
    """Rows of which each is cut into fewer chunks than there are alternatives, the largest of them all in one chunk."""
    rng = np.random.default_rng(wl)
    rows, classes = 60, 100003 if wl != 8 else 200003
    x = _logits(rng, rows, classes, wl, _fl(wl))
    top = 100 if wl == 8 else 3000
    x[0, :64], x[1, -64:] = top, top
    x[2, classes // 2:classes // 2 + 33] = np.arange(33)[::-1] + 60
    y = _labels(rng, rows, classes)
    _check_log_probs(x, (wl, _fl(wl)) if wl else None, y, 32)
    _check_cross_entropy(x[:3], (wl, _fl(wl)) if wl else None, y[:3], (8, 7))


def test_more_elements_than_32_bits_count():
    """The draws of rows that lie behind the first 2^32 elements; all rows but the last ones have no label."""
    rows, classes = 65560, 65537
    x = torch.zeros((rows, classes), dtype=torch.int8, device="cuda")
    rng = np.random.default_rng(4)
    last = _logits(rng, 3, classes, 8, 4)
    x[-3:] = dev(last)
    y = torch.full((rows,), -1, dtype=torch.int64, device="cuda")
    labels = np.array([5, 65536, 40000])
    y[-3:] = dev(labels)
    dl, logp = ctx().cross_entropy(x, (8, 4), y, (8, 7), seed=6, stream=7)
    g = head.gradient(last, 4, labels)
    lim = np.longdouble(128)
    t = np.floor(np.clip(g * lim, -lim, lim - 1) * 65536).astype(np.int64).ravel()
    want = np.minimum((t + orc.rounding_bits(t.size, orc.SR, 6, 7, start=(rows - 3) * classes)) >> 16, 127)
    assert np.array_equal(host(dl[-3:]).ravel(), want)
    assert not dl[-4].any() and not dl[0].any() and not logp[:-3].any()
    r = ctx().log_probs(x, (8, 4), y, topk=1)
    assert torch.equal(r["top_idx"][:-3], torch.zeros_like(r["top_idx"][:-3]))
    assert np.array_equal(host(r["top_idx"][-3:])[:, 0], last.argmax(1))
