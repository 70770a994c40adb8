"""AdamW with 8-bit states at the ends of fp32's range: what is stored of an element and done to its parameter does not depend on its
neighbours beyond the scale of its block, nor on where in a tensor it lies."""
import numpy as np
import pytest
import torch

from adamw_oracle import State8

pytestmark = pytest.mark.gpu
HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module")
def bg():
    import paper_2107_01499_amd as b
    assert torch.cuda.is_available()
    return b


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("size", [2.0 ** 9, 2.0 ** 11, 2.0 ** 31, 2.0 ** 33, 2.0 ** 40, 2.0 ** 62])
def test_one_large_second_moment_among_small_ones(bg, size, bf16):
    """A spike long ago: its first moment has decayed, the root of its second one has not.  At every place of a lane's four."""
    print("second moment %g^2, bf16 %d" % (size, bf16), flush=True)
    r = np.random.default_rng(7)
    n = 8 * 256 + 100
    vc, vs = np.zeros(n, np.uint8), np.zeros(9, np.float32)
    for block, at in enumerate([0, 1, 2, 3, 77, 142, 251, 252, 33]):
        vc[block * 256 + at], vs[block] = 126, size / 448
    p = r.standard_normal(n).astype(np.float32)
    if bf16:
        p = (p.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
    s = State8(bg, torch, p, vc=vc, vs=vs, bf16=bf16)
    for t in (1000, 1001, 1002):
        s.step((r.standard_normal(n) * 1e-3).astype(np.float32), t, **HYPER)
    assert bool(torch.isfinite(s.p).all())
