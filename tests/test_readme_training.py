"""The README's training loop, run against stand-ins for the network and the context (no GPU): what it hands to each call is what
the calls before it have left."""
import os
import types

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _loop():
    """From the first quantization of the weights to the end of its code block."""
    text = open(os.path.join(ROOT, "README.md")).read()
    blocks = [b for b in text.split("```python\n")[1:] if "precision_switch" in b]
    assert len(blocks) == 1
    code = blocks[0].split("```")[0]
    return code[code.index("net.quantize_weights()"):]


class _Net:
    """Formats of the last layer as a precision switch changes them, among them one of another storage size."""
    def __init__(self, n, classes, last):
        self.n, self.classes, self.last = n, classes, last
        self.formats = [(8, 4), (8, 6), (7, 4), (12, 8), (12, 7), (5, 2)]
        self.format, self.dropped, self.calls = self.formats.pop(0), {}, []

    def storage(self):
        return torch.int8 if self.format[0] <= 8 else torch.int16

    def quantize_weights(self, **kw):
        self.calls.append("quantize")

    def set_dropout(self, layer, p):
        self.dropped[layer] = p

    def forward(self, x, stream=0):
        self.calls.append("forward")

    def tensor(self, layer, which):
        assert layer == self.last
        return torch.zeros(self.n * self.classes, dtype=self.storage())

    def backward(self, dlogits, fl, stream=0):
        assert dlogits.wl == self.format[0] and dlogits.fl == fl and self.calls[-1] == "forward"
        self.calls.append("backward")

    def precision_switch(self, loss, stream=0):
        assert self.calls[-1] == "backward" and loss == loss
        self.calls.append("switch")
        self.format = self.formats.pop(0)
        other = types.SimpleNamespace(wl=16, fl=3)
        return [other] * self.last + [types.SimpleNamespace(wl=self.format[0], fl=self.format[1])], 0

    def update(self, lr, l1, l2, stream=0):
        assert self.calls[-1] == "switch"
        self.calls.append("update")


class _Context:
    def __init__(self, net):
        self.net, self.seen = net, []

    def _check(self, logits, f):
        assert f == self.net.format and logits.dtype == self.net.storage() and logits.shape == (self.net.n, self.net.classes)
        self.seen.append(f)

    def cross_entropy(self, logits, f, labels, fg, stream=0):
        self._check(logits, f)
        return types.SimpleNamespace(wl=fg[0], fl=fg[1]), torch.full((self.net.n,), -1.0)

    def log_probs(self, logits, f, labels, topk=0):
        assert not any(self.net.dropped.values()) and self.net.calls[-1] == "forward"
        self._check(logits, f)
        return {}


def test_the_loop_takes_the_formats_that_the_switch_leaves():
    import paper_2107_13490_amd as pkg
    n, classes, layers = 6, 10, [None] * 8
    net = _Net(n, classes, len(layers) - 1)
    ctx = _Context(net)
    y = torch.zeros(n, dtype=torch.int64)
    exec(_loop(), dict(pkg=pkg, net=net, ctx=ctx, layers=layers, n=n, batches=[(None, y)] * 4, lr=0.1, l1=0.0, l2=0.0, x=None, labels=y))
    assert ctx.seen == [(8, 4), (8, 6), (7, 4), (12, 8), (12, 7)]
    assert net.calls.count("update") == 4
