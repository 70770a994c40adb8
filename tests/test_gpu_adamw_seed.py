"""AdamW without a seed: every step rounds with other random numbers, those of its own number."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def bg():
    import paper_2107_01499_amd as b
    assert torch.cuda.is_available()
    return b


def stepped(bg, step, **kw):
    """Parameters and codes of the second moments after one step from the same state."""
    n = 5000
    r = torch.Generator(device="cuda").manual_seed(1)
    g = torch.randn(n, device="cuda", generator=r)
    p = torch.randn(n, device="cuda", generator=r).bfloat16()
    m, v = (torch.zeros(n, device="cuda").to(F8) for _ in range(2))
    scales = [torch.zeros(20, device="cuda") for _ in range(2)]
    ws = torch.empty(bg.bagua_tensor_plan_bytes([n]), dtype=torch.uint8, device="cuda")
    plan = bg.bagua_tensor_plan([g], ws, params=[p], m=[m], v=[v], m_scales=scales[:1], v_scales=scales[1:])
    bg.bagua_adamw_step(plan, step, 1e-3, **kw)
    return p.view(torch.uint16).cpu(), v.view(torch.uint8).cpu()


@pytest.mark.parametrize("step", [1, 7, (1 << 32) + 3])
def test_the_step_is_the_seed(bg, step):
    default, given = stepped(bg, step), stepped(bg, step, seed=step & 0xFFFFFFFF)
    assert all(torch.equal(a, b) for a, b in zip(default, given))


def test_steps_round_with_other_numbers(bg):
    """From the same state the roots of steps 1000000 and 1000001 are the same numbers; their codes are not."""
    a, b = (stepped(bg, 1000000 + i, eps=1e-8) for i in range(2))
    assert float((a[1] != b[1]).float().mean()) > 0.1
    assert float((a[0] != b[0]).float().mean()) > 0.1
