"""AdamW with 8-bit states, without a clipping factor to keep out what is no number: an element whose moment is not finite keeps a code that is
no number, and the scale of its block is that of the others, wherever in a row or a tensor it lies."""
import math

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


PLACES = {"one": [301], "one of each lane's four": [512, 517, 522, 527], "a lane's four": [304, 305, 306, 307], "a block": list(range(256, 512)), "the last": [-1],
          "in the cut share": [-9, -40, -41]}


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("places", list(PLACES))
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 1e20], ids=str)
def test_8_bits(bg, bad, places, bf16):
    print("8 bits, %s at %s, bf16 %d" % (bad, places, bf16), flush=True)
    r = np.random.default_rng(5)
    for n in (1024 + 60, 512 + 512):
        p = (r.standard_normal(n) + 3.0).astype(np.float32)
        if bf16:
            p = (p.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
        s = State8(bg, torch, p, bf16=bf16)
        for t in (1, 2, 3):
            g = (r.standard_normal(n) * 1e-3).astype(np.float32)
            if t == 2:
                g[PLACES[places]] = bad
            s.step(g, t, **HYPER)
        here = np.zeros(n, bool)
        here[PLACES[places]] = True
        assert np.array_equal(np.isnan(s.p.float().cpu().numpy()), here)
        assert np.array_equal(s.vc.cpu().numpy() == 127, here)
        assert bool(torch.isfinite(s.vs).all()) and bool(torch.isfinite(s.ms).all())


@pytest.mark.parametrize("n", [1, 2, 3])
def test_8_bits_few_elements(bg, n):
    for at in range(n):
        s = State8(bg, torch, np.ones(n, np.float32))
        for t in (1, 2):
            g = np.full(n, 0.5, np.float32)
            if t == 1:
                g[at] = math.nan
            s.step(g, t, **HYPER)
        assert torch.isnan(s.p).tolist() == [i == at for i in range(n)]


@pytest.mark.parametrize("bf16", [False, True])
def test_8_bits_first_moment_alone(bg, bf16):
    r = np.random.default_rng(6)
    n = 1024
    mc = r.integers(0, 127, n).astype(np.uint8)
    mc[[100, 513, 514, 767]] = [127, 255, 127, 127]
    s = State8(bg, torch, np.ones(n, np.float32), mc=mc, ms=np.full(4, 1e-4), vc=np.full(n, 100, np.uint8), vs=np.full(4, 1e-3), bf16=bf16)
    for t in (5, 6):
        s.step((r.standard_normal(n) * 1e-3).astype(np.float32), t, **HYPER)
    assert torch.isnan(s.p).nonzero().flatten().tolist() == [100, 513, 514, 767] and int((s.vc == 127).sum()) == 0
