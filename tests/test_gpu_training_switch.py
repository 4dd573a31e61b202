"""Training with dropout, the loss on the device and the precision switch in between: the loss takes the formats that the switch has
left, and every step's gradients and formats equal the oracle's."""
import numpy as np
import pytest

import paper_2107_13490_amd as pkg
from gpu_util import ctx, dev, host
from oracle import graph_oracle as go
from oracle import head_oracle as head
from oracle import net_oracle as no
from oracle import pushup_oracle as po
from paper_2107_13490_amd import ConvDesc, LayerDesc

pytestmark = pytest.mark.gpu

NODES = [go.Node(8, 8, 4, 8, relu=True, pool=True),
         go.Node(1, 1, 128, 24, 1, 1, 1, 0, relu=True, pool=False),
         go.Node(1, 1, 24, 10, 1, 1, 1, 0, relu=False, pool=False)]


@pytest.mark.parametrize("fmts,eps,wl_max", [([(8, 5), (8, 5), (8, 4)], 1e-2, 16), ([(12, 8), (9, 5), (7, 4)], 1e-3, 16), ([(14, 10), (20, 15), (16, 11)], 1e-6, 32)])
def test_loss_dropout_and_precision_switch(fmts, eps, wl_max):
    n, classes, seed, drop = 7, 10, 12, {0: 0.25, 1: 0.5}
    p = (1, 3, 1, 50, 80, 60, 0.4, eps, 4, 4, wl_max)
    rng = np.random.default_rng(seed)
    ws = [(rng.standard_normal((L.k, L.r, L.s, L.c)) * (1.5 / np.sqrt(L.r * L.s * L.c))).astype(np.float32) for L in NODES]
    wdev = [dev(w.copy()) for w in ws]
    descs = [LayerDesc(ConvDesc(n, L.h, L.w, L.c, L.k, L.r, L.s, L.stride, L.pad), int(L.relu), int(L.pool)) for L in NODES]
    net = pkg.Net(ctx(), descs, wdev, switch=pkg.SwitchParams(*p, pkg.ST_MIN), wl_max=wl_max)
    st = no.SwitchState(3, *p, strategy=po.ST_MIN, wl_cap=wl_max)
    fmts = list(fmts)
    for l, f in enumerate(fmts):
        net.set_format(l, *f)
    for l, q in drop.items():
        net.set_dropout(l, q)
    net.quantize_weights(seed=seed, stream=5)
    wq = no.quantize_weights(NODES, fmts, ws, seed, 5)
    wl, fl = fmts[-1]
    seen = set()
    for step in range(5):
        s0 = 1000 * (step + 1)
        seen.add((wl, fl))
        x = rng.standard_normal((n, 8, 8, 4)).astype(np.float32)
        y = rng.integers(-1, classes, n)
        net.forward(dev(x), seed=seed, stream=s0)
        fwd = go.forward(NODES, fmts, wq, [None] * 3, x, 1e-5, seed, s0, drop=drop)
        logits = net.tensor(2, pkg.NT_A).view(n, classes)
        assert np.array_equal(host(logits).astype(np.int64), fwd["a"][2].reshape(n, classes))
        dl, logp = ctx().cross_entropy(logits, (wl, fl), dev(y), (wl, wl - 1), seed=seed, stream=s0 + 999)
        want = head.quantize_real(head.gradient(fwd["a"][2].reshape(n, classes), fmts[-1][1], y), fmts[-1][0], fmts[-1][0] - 1, seed=seed, stream=s0 + 999)
        assert np.array_equal(host(dl).astype(np.int64), want), step
        net.backward(dl, wl - 1, seed=seed, stream=s0)
        bwd = go.backward(NODES, fmts, wq, fwd, want, fmts[-1][0] - 1, seed, s0, drop=drop)
        for l in range(3):
            assert np.array_equal(host(net.tensor(l, pkg.NT_G)).astype(np.int64), bwd["g"][l].ravel()), (step, l)
        loss = float(-logp.mean())
        report, strategy = net.precision_switch(loss, seed=seed, stream=s0)
        no.precision_switch(st, fmts, ws, bwd, fmts[-1][0] - 1, loss, seed, s0)
        assert [(r.wl, r.fl) for r in report] == fmts and strategy == st.strategy, step
        wl, fl = report[-1].wl, report[-1].fl
        net.update(0.05, 1e-5, 1e-4, seed=seed, stream=s0)
        upd, _ = go.update(NODES, fmts, ws, [None] * 3, bwd, 0.05, 1e-5, 1e-4, seed, s0)
        ws = [u["w"].reshape(w.shape) for u, w in zip(upd, ws)]
        wq = [u["q"].reshape(w.shape) for u, w in zip(upd, ws)]
        for l in range(3):
            assert np.array_equal(host(net.tensor(l, pkg.NT_QW)).astype(np.int64), upd[l]["q"]), (step, l)
    assert len(seen) >= 2, seen
    net.close()
