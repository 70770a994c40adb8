"""AdamW with 8-bit states: first moments below fp32's smallest normal number, whose loss would show in a parameter near zero, are the same
wherever an element lies: in a whole share of rows, in the cut one at a tensor's end, and beside an element that is huge."""
import numpy as np
import pytest
import torch

from adamw_oracle import State8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bg():
    import paper_2107_01499_amd as b
    assert torch.cuda.is_available()
    return b


@pytest.mark.parametrize("eps", [1e-30, 1e-13, 1e-8, 1.0])
@pytest.mark.parametrize("beta1", [0.0, 0.9])
def test_tiny_first_moments(bg, eps, beta1):
    print("eps %g beta1 %g" % (eps, beta1), flush=True)
    r = np.random.default_rng(3)
    n, k = 3 * 512 + 188, 188
    pattern = lambda: (2.0 ** r.uniform(-148, -100, k) * r.choice([-1.0, 1.0], k)).astype(np.float32)  # noqa: E731
    starts = (0, 512, 1024, 1536)
    mc, ms = np.zeros(n, np.uint8), np.zeros(7, np.float32)
    codes = r.integers(0, 127, k) + 128 * r.integers(0, 2, k)
    for a in starts:
        mc[a:a + k] = codes
        ms[a // 256] = 2.0 ** -121
    s = State8(bg, torch, np.zeros(n, np.float32), mc=mc, ms=ms)
    for t in (1, 2, 3):
        g, x = np.zeros(n, np.float32), pattern()
        for a in starts:
            g[a:a + k] = x
        g[1024 + 250] = 2.0 ** 40 * t                # a block whose first moments do not fit the short forms
        s.step(g, t, lr=1.0, beta1=beta1, beta2=0.999, eps=eps, weight_decay=0.0)
        if t == 1:                                   # (later the block of the huge element has another scale)
            for a in starts[1:]:
                assert torch.equal(s.p[a:a + k], s.p[:k])
        assert int((s.p[:k] != 0).sum()) > k // 4
