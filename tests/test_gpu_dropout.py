"""Dropout of codes: every output code equal to the oracle's."""
import numpy as np
import pytest
import torch

import paper_2107_13490_amd as pkg
from gpu_util import ctx, dev, host
from oracle import head_oracle as head

pytestmark = pytest.mark.gpu


def _np(wl):
    return np.int8 if wl <= 8 else np.int16 if wl <= 16 else np.int32


def _codes(rng, n, wl):
    """Codes over the whole range, the ends and zeros among them."""
    lim = 1 << (wl - 1)
    x = rng.integers(-lim, lim, n)
    x[rng.random(n) < 0.2] = 0
    if n > 2:
        x[0], x[1] = -lim, lim - 1
    return x.astype(_np(wl))


def _check(n, fx, fo, p, res_fmt=None, mode=pkg.SR, seed=7, stream=11, data=0):
    rng = np.random.default_rng([n, data])
    x = _codes(rng, n, fx[0])
    res = _codes(rng, n, res_fmt[0]) if res_fmt else None
    got = ctx().dropout(dev(x), fx, p, fo=fo, res=dev(res) if res_fmt else None, fres=res_fmt, mode=mode, seed=seed, stream=stream)
    want = head.dropout(x, fx[1], p, fo[0], fo[1], mode=mode, seed=seed, stream=stream, res=res, fl_res=res_fmt[1] if res_fmt else 0)
    got = host(got)
    assert got.dtype == _np(fo[0]) and np.array_equal(got, want)


@pytest.mark.parametrize("n", [1, 7, 8, 9, 16, 255, 2048, 2049, 70001])
@pytest.mark.parametrize("fx,fo", [((8, 4), (8, 4)), ((16, 12), (16, 11)), ((8, 4), (16, 9)), ((16, 9), (8, 4)), ((4, 3), (4, 1))])
def test_sizes(n, fx, fo):
    _check(n, fx, fo, 0.3)


@pytest.mark.parametrize("p", [0.0, 0.5 / 65536, 1 / 65536, 0.1, 0.25, 0.5, 0.75, 0.99, 65535 / 65536])
@pytest.mark.parametrize("fx,fo", [((8, 4), (8, 4)), ((16, 10), (16, 12)), ((24, 20), (24, 19)), ((32, 20), (32, 20))])
def test_probabilities(p, fx, fo):
    _check(5003, fx, fo, p)


@pytest.mark.parametrize("fx,fo", [((8, 0), (8, 15)), ((16, 31), (16, 0)), ((8, 20), (8, 0)), ((16, 17), (8, 0)), ((32, 31), (8, 0)),
                                   ((32, 0), (32, 15)), ((16, 3), (32, 18)), ((2, 0), (2, 0)), ((20, 10), (8, 2)), ((8, 2), (20, 10))])
@pytest.mark.parametrize("mode", [pkg.SR, pkg.RN_HALF_UP])
def test_formats(fx, fo, mode):
    _check(4099, fx, fo, 0.2, mode=mode)


@pytest.mark.parametrize("fx,res,fo", [((8, 4), (8, 4), (8, 4)), ((8, 4), (16, 9), (16, 10)), ((16, 9), (8, 3), (8, 3)),
                                       ((16, 12), (16, 12), (16, 12)), ((16, 12), (32, 5), (16, 12)), ((32, 28), (8, 4), (8, 4)),
                                       ((32, 16), (32, 0), (32, 31)), ((8, 4), (8, 0), (8, 15)), ((16, 16), (16, 0), (16, 31)),
                                       ((4, 3), (8, 4), (32, 18))])
@pytest.mark.parametrize("n", [5, 8192, 10007])
def test_residuals(fx, res, fo, n):
    _check(n, fx, fo, 0.1, res_fmt=res)


def test_wide_seeds_and_streams():
    _check(4001, (8, 4), (8, 4), 0.4, seed=(1 << 63) + 12345, stream=(1 << 40) + 3)


@pytest.mark.parametrize("lo", [1, 2, 3, 5])
def test_unaligned_views(lo):
    rng = np.random.default_rng(lo)
    for wl in (8, 16, 24):
        x, res = _codes(rng, 6007, wl), _codes(rng, 6007, wl)
        out = torch.zeros(6007, dtype=ctx().storage_dtype(wl), device="cuda")
        ctx().dropout(dev(x)[lo:6000], (wl, 4), 0.3, res=dev(res)[2 * lo:6000 + lo], fres=(wl, 4), seed=5, stream=6, out=out[lo + 1:6001])
        got = host(out)
        want = head.dropout(x[lo:6000], 4, 0.3, wl, 4, seed=5, stream=6, res=res[2 * lo:6000 + lo], fl_res=4)
        assert np.array_equal(got[lo + 1:6001], want)
        assert not got[:lo + 1].any() and not got[6001:].any()


def test_in_place():
    x = _codes(np.random.default_rng(1), 30001, 16)
    t = dev(x)
    assert ctx().dropout(t, (16, 12), 0.5, fo=(16, 11), seed=2, stream=3, out=t) is t
    assert np.array_equal(host(t), head.dropout(x, 12, 0.5, 16, 11, seed=2, stream=3))


def test_gradient():
    """The output is affine in x for given draws where the scale is a whole number of output steps (p = 1/2): differences
    of outputs are the call on the differences, and that call is the gradient.  Dropped elements have gradient 0."""
    rng = np.random.default_rng(3)
    x, h = rng.integers(-30, 30, 20000).astype(np.int8), rng.integers(-30, 30, 20000).astype(np.int8)
    c = ctx()
    y = [host(c.dropout(dev(v), (8, 4), 0.5, seed=9, stream=4)).astype(int) for v in (x, (x + h).astype(np.int8))]
    g = host(c.dropout(dev(h), (8, 4), 0.5, seed=9, stream=4)).astype(int)
    assert np.array_equal(y[1] - y[0], g)
    assert np.array_equal(g == 0, (h == 0) | (host(c.dropout(dev(np.ones_like(x)), (8, 4), 0.5, seed=9, stream=4)) == 0))


def test_captured_and_replayed():
    rng = np.random.default_rng(8)
    x, r = _codes(rng, 12345, 8), _codes(rng, 12345, 8)
    tx, tr, out = dev(x), dev(r), torch.empty(12345, dtype=torch.int8, device="cuda")
    stream = torch.cuda.Stream()
    c = pkg.Context(stream=stream)
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        c.dropout(tx, (8, 4), 0.1, res=tr, fres=(8, 4), seed=1, stream=2, out=out)
    for k in range(3):
        x = _codes(np.random.default_rng(k), 12345, 8)
        tx.copy_(dev(x))
        out.zero_()
        graph.replay()
        assert np.array_equal(host(out), head.dropout(x, 4, 0.1, 8, 4, seed=1, stream=2, res=r, fl_res=4))


def test_empty():
    assert ctx().dropout(torch.empty(0, dtype=torch.int8, device="cuda"), (8, 4), 0.5).numel() == 0


def test_refusals():
    c = ctx()
    x = torch.zeros(64, dtype=torch.int8, device="cuda")
    for bad in (dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(p=0.999999), dict(fx=(8, 32)), dict(fo=(33, 0)), dict(fx=(8, 0), fo=(8, 16)),
                dict(mode=2), dict(res=x, fres=(8, 5))):
        with pytest.raises(pkg.AdaptError):
            c.dropout(x, **{"fx": (8, 4), "p": 0.5, **bad})
    with pytest.raises(ValueError):
        c.dropout(x, (16, 4), 0.5)
    with pytest.raises(ValueError):
        c.dropout(x[::2], (8, 4), 0.5)
    with pytest.raises(ValueError):
        c.dropout(x.cpu(), (8, 4), 0.5)
    with pytest.raises(ValueError):
        c.dropout(x, (8, 4), 0.5, res=x[:32], fres=(8, 4))
    with pytest.raises(ValueError):
        c.dropout(x, (8, 4), 0.5, out=torch.zeros(64, dtype=torch.int16, device="cuda"))


def test_more_elements_than_32_bits_count():
    n, tail = (1 << 32) + 1003, 5001
    rng = np.random.default_rng(5)
    last = _codes(rng, tail, 8)
    x = torch.ones(n, dtype=torch.int8, device="cuda")
    x[-tail:] = dev(last)
    out = ctx().dropout(x, (8, 4), 0.25, seed=8, stream=9)
    from oracle import fxp_oracle as orc
    bits = orc.rounding_bits(tail, orc.SR, 8, 9, start=n - tail)
    assert np.array_equal(host(out[-tail:]), head.dropout_with_bits(last, 4, 0.25, 8, 4, bits))
    bits = orc.rounding_bits(4096, orc.SR, 8, 9)
    assert np.array_equal(host(out[:4096]), head.dropout_with_bits(np.ones(4096), 4, 0.25, 8, 4, bits))
