"""Balance loss over launches of many groups: where the groups' sums are put together in two steps, where the last cluster of groups is not
whole, and where every wave has several tiles, in every type and width of a row.  The bound on the probabilities' sums is far below what a
group or a tile adds to them."""
import numpy as np
import pytest
import torch

from test_gpu_balance import U, buffers, check_gradient, inputs, stats, truth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bg():
    import paper_2107_01499_amd as b
    assert torch.cuda.is_available()
    return b


CASES = [
    # more than 256 experts, more than 32 groups of 4 to 16 rows
    (257, "f32", [1100], None), (257, "bf16", [2200], 0.2), (300, "f16", [20000, 1, 0, 777], None), (512, "bf16", [17000], 0.3), (513, "f32", [5000, 300], 0.3),
    (1024, "f16", [9000], None), (1025, "bf16", [530], None), (1025, "f32", [300], 0.1), (1500, "bf16", [2100, 3], 0.5), (2048, "f32", [2500, 5], None),
    (2048, "f16", [3000], 0.2),
    # several tiles a wave
    (1, "bf16", [1100000], None), (2, "bf16", [600000], 0.1), (3, "f32", [300000, 0, 5], 0.5), (8, "bf16", [1100000, 7], None), (8, "f32", [70000] * 8, 0.1),
    (60, "f32", [70000, 130], 0.2), (64, "f16", [140000], None), (64, "bf16", [40000] * 5, 0.2), (100, "f16", [66000], 0.2), (128, "bf16", [66000, 500], None),
    (160, "f32", [20000], 0.2), (256, "f16", [34000], None)]


@pytest.mark.parametrize("experts,dtype,tokens,masked", CASES, ids=lambda v: str(v).replace(" ", ""))
def test_many_groups(bg, experts, dtype, tokens, masked):
    print("balance experts=%d %s tokens=%s masked=%s" % (experts, dtype, tokens, masked), flush=True)
    top, n = min(experts, 3), sum(tokens)
    s = inputs(tokens, experts, top, dtype, experts + n, masked=masked)
    b = buffers(bg, experts)
    stats(bg, s, b, 1.0)
    counts, valid, prob, loss, weight, reach = truth(s, experts, top, 1.0)
    assert np.array_equal(b["counts"].cpu().numpy(), np.append(counts, valid))
    # a probability is off by (3 reach + 60) U; the sums over rows are chains in fp32 within a group only: at least 2048 waves share the rows
    # where there are more than these, a wave adds a tile's rows of a lane, four at most, one after another, 6 times across its lanes, and a
    # group adds 16 waves; the rest is in 64 bits
    bound = (3 * reach + 60 + 4 * (1 + (n + len(tokens)) / 2048) + 24) * U
    assert bound < 0.4 / 256                             # a group's share of the sums
    got = b["prob"].double().cpu().numpy()
    assert np.all(np.abs(got - prob) <= bound * prob + 2.0 ** -100), np.max(np.abs(got - prob) / np.maximum(prob, 1e-30))
    assert np.all(np.abs(b["weight"].double().cpu().numpy() - weight) <= 2 * U * weight) and abs(float(b["loss"]) - loss) <= (bound + 4 * U) * loss
    again = dict(buffers(bg, experts), ws=b["ws"])
    stats(bg, s, again, 1.0)
    assert all(torch.equal(b[k], again[k]) for k in ("counts", "prob", "loss", "weight"))


@pytest.mark.parametrize("experts,dtype,tokens,masked", [(260, "f32", [66000], 0.2), (520, "f16", [65700, 3], None)], ids=str)
def test_gradient_of_many_rows(bg, experts, dtype, tokens, masked):
    print("gradient experts=%d %s tokens=%s masked=%s" % (experts, dtype, tokens, masked), flush=True)
    s = inputs(tokens, experts, 1, dtype, experts, masked=masked)
    check_gradient(bg, s, experts, dtype, torch.rand(experts, device="cuda"), torch.tensor([3.0], device="cuda"))
