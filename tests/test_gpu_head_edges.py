"""Log probabilities and cross entropy at the ends of their ranges, on the GPU against the oracle."""
import numpy as np
import pytest

from gpu_util import ctx, dev, host
from oracle import fxp_oracle as orc
from oracle import head_oracle as head

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
