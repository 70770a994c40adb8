"""Balance loss of rows of finite logits of any magnitude: the softmax is that of the differences within a row, however far from zero the row
lies.  Statistics and gradient against the formulas in 64 bits on the same numbers."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
# fill values that masks are made with, and both sides of powers of two
SIZES = [1e3, 2.0 ** 15, 2.0 ** 19, 2.0 ** 20 - 4096, 2.0 ** 20, 2.0 ** 20 + 8192, 2.0 ** 21, 1e8, 1e9, 3e9, 1e10, 1e12, 1e20, 1e30, 3e37, 2.0 ** 126, 1.5e38, 3e38]


@pytest.fixture(scope="module")
def bg():
    import paper_2107_01499_amd as b
    assert torch.cuda.is_available()
    return b


def rows(size, experts, dtype):
    """Rows around `size`: all alike, one a step of the type above or below the others, several steps, one against zeros, one against its
    negative."""
    x = torch.full((7, experts), size, dtype=torch.float64).to(TYPES[dtype])
    step = 2.0 ** (math.floor(math.log2(abs(float(x[0, 0])))) - {"f32": 23, "bf16": 7, "f16": 10}[dtype])
    x[1, experts // 2] += step
    x[2, 0] -= step
    x[3] -= (step * (torch.arange(experts) % 5)).to(x.dtype)
    x[4, 1:] = 0.0
    x[5, :-1] = -x[5, :-1]
    x[6, 1:3] = 0.0
    return x


@pytest.mark.parametrize("experts", [1, 2, 6, 8, 24, 64, 100, 256, 300, 600, 1100])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_rows_of_any_magnitude(bg, dtype, experts):
    for sign in (1.0, -1.0):
        for size in SIZES:
            if dtype == "f16" and size > 2.0 ** 15:
                continue
            print("rows around %g, %d experts, %s" % (sign * size, experts, dtype), flush=True)
            x = rows(sign * size, max(experts, 3), dtype)[:, :experts].contiguous()
            assert bool(torch.isfinite(x).all())
            n, top = x.shape[0], min(2, experts)
            ids = torch.arange(n * top).view(n, top) % experts
            z = x.double().numpy()
            z = z - z.max(1, keepdims=True)
            p = np.exp(z)
            p /= p.sum(1, keepdims=True)
            xs, ids = x.cuda(), ids.cuda()
            counts, prob = torch.zeros(experts + 1, dtype=torch.int32, device="cuda"), torch.zeros(experts, device="cuda")
            loss, weight = torch.zeros(1, device="cuda"), torch.zeros(experts, device="cuda")
            ws = torch.zeros(bg.bagua_balance_workspace_bytes(experts), dtype=torch.uint8, device="cuda")
            bg.bagua_balance_stats([xs], [ids], None, counts, prob, ws, 1.0, loss, weight)
            # the exponent's argument is off by 3 U of itself and the exponential, its sum (32 in a lane, 6 exchanges) and the reciprocal by 60 U;
            # the row's sum by as much of each of its terms, the sum over the rows by n U; of an argument beyond 120 fp32 holds nothing
            off = (3 * np.minimum(-z, 120.0) + 60) * U
            off = p * (off + (p * off).sum(1, keepdims=True))
            bound = (off + n * U * p).sum(0) + 2.0 ** -100
            assert np.all(np.abs(prob.double().cpu().numpy() - p.sum(0)) <= bound)
            w = weight.double().cpu().numpy()
            want = float((w * p.sum(0)).sum())
            assert abs(float(loss) - want) <= (bound * w).sum() + 4 * U * want
            w = torch.rand(experts, device="cuda", generator=torch.Generator(device="cuda").manual_seed(experts))
            out = [torch.full_like(xs, 9.0)]
            bg.bagua_balance_grad([xs], None, w, None, out)
            w = w.double().cpu().numpy()
            dot = (p * w).sum(1, keepdims=True)
            want = p * (w - dot)
            bound = off * (w + dot) + p * (off * w).sum(1, keepdims=True) + 150 * U * p * (w + dot)
            assert np.all(np.abs(out[0].double().cpu().numpy() - want) <= bound + 1.01 * HALF_ULP[dtype] * np.abs(want) + 2.0 ** -24)
