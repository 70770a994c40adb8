"""One AdamW step with 8-bit states in NumPy, operation by operation, on the stored codes and scales.  The first moment and the quotient are
held with fp32's 24 bits and an exponent without a lower end, as the step defines them; everything else in fp32."""
import math

import numpy as np

from test_gpu_tensors import VALUES, decode, hashes

LONG = np.longdouble


def round24(x):
    """To the nearest number of 24 bits (ties to even), whatever its exponent."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(np.ldexp(m, 24)), e - 24)


def largest(x):
    """The largest finite magnitude of each block of 256, in fp32."""
    pad = np.zeros(-(-x.size // 256) * 256, np.float32)
    with np.errstate(over="ignore", under="ignore"):
        pad[:x.size] = np.where(np.isfinite(x), np.abs(x), 0)
    return pad.reshape(-1, 256).max(1)


def scale_of(most):
    """Of each block, and its reciprocal."""
    s = most * np.float32(1.0 / 448.0)
    s = np.where(s >= np.float32(2.0 ** -126), s, np.float32(0))
    with np.errstate(divide="ignore"):
        return s, np.where(s > 0, np.float32(1) / s, np.float32(0)).astype(np.float32)


def nearest(y):
    """Codes of the values next to y; that of what is no number: 127."""
    a = np.where(np.isfinite(y), np.abs(y).astype(np.float64), 0.0)
    hi = np.searchsorted(VALUES, a).clip(0, 126)
    lo = (hi - 1).clip(0)
    up = (VALUES[hi] - a < a - VALUES[lo]) | ((VALUES[hi] - a == a - VALUES[lo]) & (hi % 2 == 0))
    return np.where(np.isfinite(y), np.where(up, hi, lo), 127).astype(np.uint8)


def values(codes, scale):
    """What the codes stand for; code 127 for no number."""
    x = decode(np.where(codes % 128 == 127, 0, codes), scale)
    return np.where(codes % 128 == 127, np.float32(np.nan), x)


def step8(p, g, mc, ms, vc, vs, t, seed, lr, beta1, beta2, eps, weight_decay, tensor=0, bf16=False):
    """p, g in fp32 (as widened), codes and scales of both moments: p, codes and scales after the step.  p of bf16: the upper halves' bits."""
    f, n = np.float32, p.size
    with np.errstate(all="ignore"):
        m = LONG(1) * values(mc, np.ones_like(ms)) * np.repeat(ms, 256)[:n]
        m = round24(round24(round24(m) * f(beta1)) + round24(LONG(1) * g * f(1.0 - beta1)))
        m = np.where(np.isnan(g) | np.isinf(g), LONG(1) * g, m)
        v = values(vc, vs)
        v = v * v
        v = v * f(beta2) + (g * g) * f(1.0 - beta2)
        r = np.sqrt(v)
        b = r * f(1.0 / math.sqrt(1.0 - beta2 ** t)) + f(eps)
        u = np.where(np.isfinite(b), round24(m / b), np.where(np.isfinite(m) & np.isinf(b), LONG(0), LONG(np.nan)))
        p = p - ((u * f(lr / (1.0 - beta1 ** t))).astype(f) + p * f(lr * weight_decay))
        h, h2 = hashes(n, tensor, seed)
        if bf16:
            bits = ((p.view(np.uint32).astype(np.uint64) + (h2 >> np.uint32(16))) >> np.uint64(16)).astype(np.uint32) << np.uint32(16)
            p = np.where(np.isnan(p), p, bits.view(f))
        ms, inverse = scale_of(largest(m))
        inverse = np.repeat(inverse, 256)[:n]
        mc = nearest(np.where(np.isfinite(m), (m * inverse).astype(f), f(np.nan))) + np.where(np.signbit(m), 128, 0).astype(np.uint8)
        vs, inverse = scale_of(largest(r))
        y = r * np.repeat(inverse, 256)[:n]
        c = ((y * f(2.0 ** -120)).view(np.uint32) + (h >> np.uint32(12))) >> np.uint32(20)
        vc = np.where(np.isfinite(r), np.where(r > 0, c.clip(1, 126), 0), 127).astype(np.uint8)
    return p, mc, ms, vc, vs


class State8:
    """A tensor with its states on the GPU, and their copies in NumPy."""

    def __init__(self, bg, torch, p, mc=None, ms=None, vc=None, vs=None, bf16=False):
        n = self.n = p.size
        blocks = -(-n // 256)
        self.torch, self.bf16, self.bg = torch, bf16, bg
        zero = lambda x, count, dtype: np.zeros(count, dtype) if x is None else x.astype(dtype)  # noqa: E731
        self.host = [p.astype(np.float32), zero(mc, n, np.uint8), zero(ms, blocks, np.float32), zero(vc, n, np.uint8), zero(vs, blocks, np.float32)]
        gpu = [torch.from_numpy(x.copy()).cuda() for x in self.host]
        if bf16:
            gpu[0] = (gpu[0].view(torch.int32) >> 16).to(torch.int16).view(torch.bfloat16)
        self.p, self.mc, self.ms, self.vc, self.vs = gpu
        self.g = torch.zeros(n, device="cuda")
        ws = torch.empty(bg.bagua_tensor_plan_bytes([n]), dtype=torch.uint8, device="cuda")
        f8 = torch.float8_e4m3fn
        self.plan = bg.bagua_tensor_plan([self.g], ws, params=[self.p], m=[self.mc.view(f8)], v=[self.vc.view(f8)], m_scales=[self.ms], v_scales=[self.vs])

    def step(self, g, t, **hyper):
        """Both sides; everything equal bit for bit (what is no number: no number on both).  The bits of p before and after are returned."""
        torch = self.torch
        self.g.copy_(torch.from_numpy(g))
        self.bg.bagua_adamw_step(self.plan, t, seed=t, **hyper)
        self.host = list(step8(self.host[0], g, *self.host[1:], t, t, bf16=self.bf16, **hyper))
        for what, x, want in zip(("p", "m", "m_scale", "v", "v_scale"), (self.p, self.mc, self.ms, self.vc, self.vs), self.host):
            got = x.float().cpu().numpy() if what == "p" else x.cpu().numpy()
            if want.dtype == np.uint8:
                wrong = (got != want) & ~((got % 128 == want % 128) & ((want % 128 == 127) | (want % 128 == 0)))
            else:
                wrong = (got.view(np.uint32) != want.view(np.uint32)) & ~(np.isnan(got) & np.isnan(want))
            at = np.flatnonzero(wrong)
            assert at.size == 0, "%s: %d of %d differ, first at %d: %r, expected %r" % (what, at.size, got.size, at[0], got[at[0]], want[at[0]])
