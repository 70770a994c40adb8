"""What the entry points for many tensors and for the balance loss refuse, from the host alone: no case here reaches a launch."""
import ctypes
import math

import pytest

OK, INVALID, ALIGN, UNSUPPORTED = 0, 1, 2, 4
# far-apart, aligned addresses that nothing looks at
G, P, M, V, MS, VS, C, W = (0x100000000 * i for i in range(1, 9))


@pytest.fixture(scope="module")
def bg():
    import paper_2107_01499_amd as b
    return b


def ptrs(*a):
    return (ctypes.c_void_p * len(a))(*a)


def sizes(*n):
    return (ctypes.c_size_t * len(n))(*n)


def test_workspace_sizes(bg):
    assert bg.bagua_tensor_plan_bytes([]) == 0
    assert bg.bagua_tensor_plan_bytes([0]) >= 80
    small, large = bg.bagua_tensor_plan_bytes([1024]), bg.bagua_tensor_plan_bytes([1024 * 1000])
    assert abs(large - small - 4 * 999) <= 16 and small % 16 == 0
    assert bg.bagua_tensor_plan_bytes([1 << 45]) == 0
    assert bg.bagua_balance_workspace_bytes(0) == 0 == bg.bagua_balance_workspace_bytes(2049)
    assert bg.bagua_balance_workspace_bytes(2048) > bg.bagua_balance_workspace_bytes(8) > 64


PLAN = dict(numel=sizes(1000), T=1, grad=ptrs(G), grad_type=0, param=ptrs(P), param_type=0, m=ptrs(M), v=ptrs(V), bits=32, ms=None, vs=None, copy=None,
            copy_type=0, decay=None, ws=W, bytes=1 << 20)


def plan(bg, out=True, **kw):
    a = dict(PLAN, **kw)
    s = bg.binding._PlanStruct()
    return bg.binding.raw().bagua_tensor_plan(a["numel"], a["T"], a["grad"], a["grad_type"], a["param"], a["param_type"], a["m"], a["v"], a["bits"], a["ms"],
                                              a["vs"], a["copy"], a["copy_type"], a["decay"], a["ws"], a["bytes"], ctypes.addressof(s) if out else None, None)


EIGHT = dict(bits=8, ms=ptrs(MS), vs=ptrs(VS))


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), INVALID), (dict(numel=None), INVALID), (dict(grad=None), INVALID), (dict(ws=None), INVALID), (dict(out=False), INVALID),
    (dict(grad_type=3), INVALID), (dict(grad_type=-1), INVALID), (dict(m=None), INVALID), (dict(v=None), INVALID), (dict(bits=16), INVALID),
    (dict(bits=0), INVALID), (dict(param_type=2), INVALID), (dict(param=None), INVALID), (dict(bits=8), INVALID), (dict(ms=ptrs(MS)), INVALID),
    (dict(EIGHT, vs=None), INVALID), (dict(param_type=1, copy=ptrs(C), copy_type=1), INVALID), (dict(copy=ptrs(C), copy_type=0), INVALID),
    (dict(param_type=1, grad_type=2), INVALID), (dict(grad=ptrs(None)), INVALID), (dict(param=ptrs(None)), INVALID), (dict(bytes=64), INVALID),
    (dict(decay=(ctypes.c_float * 1)(math.inf)), INVALID), (dict(numel=sizes(1 << 42)), UNSUPPORTED), (dict(numel=sizes(1 << 63)), UNSUPPORTED),
    (dict(ws=W + 8), ALIGN), (dict(grad=ptrs(G + 2)), ALIGN), (dict(grad=ptrs(G + 1), grad_type=1), ALIGN), (dict(param=ptrs(P + 2)), ALIGN),
    (dict(param=ptrs(P + 1), param_type=1), ALIGN), (dict(v=ptrs(V + 2)), ALIGN), (dict(EIGHT, ms=ptrs(MS + 2)), ALIGN),
    (dict(copy=ptrs(C + 1), copy_type=1), ALIGN), (dict(param=ptrs(G)), INVALID), (dict(m=ptrs(P + 3996)), INVALID), (dict(EIGHT, m=ptrs(V + 999)), INVALID),
    (dict(EIGHT, vs=ptrs(MS + 12)), INVALID), (dict(copy=ptrs(G + 2000), copy_type=1), INVALID), (dict(ws=P + 16), INVALID)])
def test_plan_refuses(bg, kw, status):
    assert plan(bg, **kw) == status


def test_calls_refuse(bg):
    lib = bg.binding.raw()
    at = lambda **kw: bg.binding._PlanStruct(**dict(dict(workspace=W, tiles=1, tensors=1, state_bits=32), **kw))  # noqa: E731
    norm = lambda s, scale=1.0, most=1.0, out=C: lib.bagua_grad_norm(ctypes.addressof(s) if s else None, scale, most, out, None)  # noqa: E731
    bad = [at(workspace=None), at(workspace=W + 4), at(tensors=0), at(tiles=1 << 40), at(grad_type=7)]
    for s in [None] + bad:
        assert norm(s) == INVALID
        assert lib.bagua_adamw_step(ctypes.addressof(s) if s else None, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, None, 0, None) == INVALID
    assert norm(at(), out=None) == INVALID and norm(at(), out=C + 2) == ALIGN
    for scale, most in ((math.nan, 1.0), (math.inf, 1.0), (1.0, math.nan), (1.0, -1.0)):
        assert norm(at(), scale, most) == INVALID
    good = [1, 1e-3, 0.9, 0.999, 1e-8, 0.0, None, 0]
    for i, x, status in ((0, 0, INVALID), (1, math.nan, INVALID), (2, 1.0, INVALID), (2, -0.1, INVALID), (3, 1.0, INVALID), (3, math.nan, INVALID),
                         (4, -1.0, INVALID), (4, math.inf, INVALID), (5, math.inf, INVALID), (6, C + 2, ALIGN)):
        a = list(good)
        a[i] = x
        s = at()
        assert lib.bagua_adamw_step(ctypes.addressof(s), *a, None) == status
    s = at(state_bits=0)
    assert lib.bagua_adamw_step(ctypes.addressof(s), *good, None) == INVALID
    s = at(tiles=0)                                       # nothing but empty tensors: nothing to launch
    assert lib.bagua_adamw_step(ctypes.addressof(s), *good, None) == OK


STATS = dict(dtype=0, logits=ptrs(G), ld=8, tokens=sizes(10), k=1, experts=8, ids=ptrs(P), id_bytes=8, ids_ld=2, top=2, mask=None, counts=M, prob=V, alpha=0.01,
             loss=MS, weight=VS, ws=W, bytes=1 << 20)
GRAD = dict(dtype=0, logits=ptrs(G), ld=8, tokens=sizes(10), k=1, experts=8, mask=None, weight=VS, up=None, out=ptrs(P), ld_out=8)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), INVALID), (dict(logits=None), INVALID), (dict(logits=ptrs(None)), INVALID), (dict(tokens=None), INVALID), (dict(k=0), INVALID),
    (dict(k=33), INVALID), (dict(experts=0), INVALID), (dict(ld=7), INVALID), (dict(experts=2049, ld=2049), UNSUPPORTED), (dict(tokens=sizes(1 << 31)), UNSUPPORTED),
    (dict(tokens=sizes(1 << 30)), UNSUPPORTED), (dict(ids=None), INVALID), (dict(ids=ptrs(None)), INVALID), (dict(id_bytes=2), INVALID), (dict(top=0), INVALID),
    (dict(top=9, ids_ld=9), INVALID), (dict(ids_ld=1), INVALID), (dict(ld=1 << 50), UNSUPPORTED), (dict(ids_ld=1 << 50), UNSUPPORTED), (dict(mask=ptrs(None)), INVALID),
    (dict(counts=None), INVALID), (dict(prob=None), INVALID), (dict(loss=None), INVALID), (dict(weight=None), INVALID), (dict(alpha=math.nan), INVALID),
    (dict(ws=None), INVALID), (dict(bytes=100), INVALID), (dict(ws=W + 8), ALIGN), (dict(logits=ptrs(G + 2)), ALIGN), (dict(dtype=1, logits=ptrs(G + 1)), ALIGN),
    (dict(ids=ptrs(P + 4)), ALIGN), (dict(ids=ptrs(P + 2), id_bytes=4), ALIGN), (dict(counts=M + 2), ALIGN), (dict(prob=V + 1), ALIGN), (dict(prob=M + 32), INVALID),
    (dict(counts=G + 316), INVALID), (dict(weight=V), INVALID), (dict(ws=V), INVALID), (dict(loss=P + 156), INVALID)])
def test_statistics_refuse(bg, kw, status):
    a = dict(STATS, **kw)
    assert bg.binding.raw().bagua_balance_stats(*[a[k] for k in STATS], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=-1), INVALID), (dict(weight=None), INVALID), (dict(out=None), INVALID), (dict(out=ptrs(None)), INVALID), (dict(ld_out=7), INVALID),
    (dict(ld_out=1 << 50), UNSUPPORTED), (dict(out=ptrs(G)), INVALID), (dict(out=ptrs(G + 316)), INVALID), (dict(weight=P), INVALID), (dict(out=ptrs(P + 1)), ALIGN),
    (dict(weight=VS + 2), ALIGN), (dict(up=C + 2), ALIGN), (dict(mask=ptrs(None)), INVALID), (dict(tokens=sizes(0), logits=ptrs(None), out=ptrs(None)), OK)])
def test_gradient_refuses(bg, kw, status):
    a = dict(GRAD, **kw)
    assert bg.binding.raw().bagua_balance_grad(*[a[k] for k in GRAD], None) == status


def test_calls_that_are_not_ordinary_are_declined(bg):
    """The host extension's part of these calls leaves what it does not know to the general path, and does nothing."""
    import torch
    native = bg.binding._native
    x, ids, c, p = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int64), torch.zeros(9, dtype=torch.int32), torch.zeros(8)
    for f, count in ((native.grad_norm, 5), (native.adamw_step, 10), (native.balance_stats, 10), (native.balance_grad, 6)):
        for n in (0, count - 1, count, count + 1):
            assert f(*[None] * n) is False
    assert native.balance_stats([x], [ids], None, c, p, c, 0.01, None, None, None) is False        # not on the GPU
    assert native.balance_grad([x], None, p, None, [x], None) is False
    assert native.grad_norm(0, p, 1.0, 1.0, None) is False and native.grad_norm("plan", p, 1.0, 1.0, None) is False
    assert native.tensor_sizes((x,)) is False and native.tensor_sizes([x, 3]) is False
    assert native.tensor_sizes([x, ids]) == bytes(sizes(32, 8))
    assert native.tensor_addresses([x], x, bytes(sizes(32)), 1, False) is False                    # not on the GPU
    assert native.tensor_addresses([x], x, b"", 1, False) is False and native.tensor_addresses([x], x, bytes(sizes(32)), 0, False) is False
    with pytest.raises(ValueError, match="contiguous GPU tensor"):
        bg.bagua_tensor_plan([x], torch.zeros(10, dtype=torch.uint8))
    with pytest.raises(ValueError, match="expected GPU tensors"):
        bg.bagua_balance_grad([x], None, p, None, [x])


@pytest.mark.parametrize("scale", [-1.0, -1e-30, -math.inf])
def test_norm_refuses_a_scale_below_zero(bg, scale):
    """The norm would come out negative, and the factor would turn the gradients around."""
    s = bg.binding._PlanStruct(workspace=W, tiles=1, tensors=1, state_bits=32)
    assert bg.binding.raw().bagua_grad_norm(ctypes.addressof(s), scale, 1.0, C, None) == INVALID
