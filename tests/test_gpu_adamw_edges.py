"""GPU: AdamW where its denominator is zero, tiny or huge, against float64.  U = 2^-24 is the half step of float32."""
import numpy as np
import pytest
import torch

from paper_1806_04090_amd import binding
from gpu_common import ctx

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
B1, B2 = 0.9, 0.999


def normal(n, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(n, generator=g, device="cuda")


# 1e-50 is zero in float32, 1e-40 and 1e-45 are below its smallest normal number 2^-126
TINY = [0.0, 1e-50, 1e-45, 1e-40, 2.0 ** -126, 1e-8]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", TINY)
def test_an_element_without_a_gradient_does_not_move(bits, eps):
    n = 1300
    p, g = normal(n, 1), normal(n, 2)
    g[::3] = 0.0
    g[512:1024] = 0.0
    none = g == 0
    before = p.clone()
    s = binding.alloc_adamw_state(n, bits, "cuda")
    plan = binding.AdamwPlan(ctx(), [p], [g], [s], weight_decay=0.5)
    for t in range(1, 4):
        binding.atomo_adamw_step(ctx(), plan, 0.1, B1, B2, eps, step=t)
        assert torch.isfinite(p).all()
        # nothing but the decay: its factor is rounded, its product, and the difference
        want = before[none].double() * 0.95 ** t
        assert ((p[none].double() - want).abs() <= 3 * U * t * before[none].double().abs()).all()
        if t == 1:                                               # the others move by the rate (its error is far below a thousandth)
            off = (p.double() - before.double() * 0.95 + 0.1 * g.double().sign())[~none]
            assert (off.abs() <= 1e-3 * 0.1).all()
        assert (s.m[none] == 0).all() and (s.v[none] == 0).all()


def state_of(bits, m, n):
    """States of n elements that all have this m (a power of two) and a v of zero."""
    s = binding.alloc_adamw_state(n, bits, "cuda")
    if bits == 32:
        s.m.fill_(m)
    else:
        s.m.fill_(0x70)                                          # exponent 14, the largest of a block: 2^7 in units of 2^(E - 7)
        s.m_scale.fill_(int(np.log2(m)) + 127)
        assert (binding.atomo_state8_unpack(ctx(), "m", s.m, s.m_scale) == m).all()
    return s


# with v = 0 and g = 0 the update is lr / (1 - b1) * b1 m / eps
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("m, eps", [(2.0 ** -100, 1e-40), (-(2.0 ** -100), 3e-39), (2.0 ** -120, 1e-45), (2.0 ** -60, 2.0 ** -126), (2.0 ** 5, 1e-8),
                                    (2.0 ** 100, 1e37), (2.0 ** 120, 1e38), (2.0 ** 120, 3e38)])
def test_a_denominator_of_eps_alone(bits, m, eps):
    n = 700
    s = state_of(bits, abs(m), n)
    if m < 0:
        s.m.neg_() if bits == 32 else s.m.bitwise_or_(0x80)
    p = torch.zeros(n, device="cuda")
    eps32 = float(np.float32(eps))
    lr = 0.1 * eps32 / abs(m)
    plan = binding.AdamwPlan(ctx(), [p], [torch.zeros(n, device="cuda")], [s])
    binding.atomo_adamw_step(ctx(), plan, lr, B1, B2, eps, step=1)
    want = -lr / (1 - B1) * B1 * m / eps32
    # b1 and its product, the quotient (its reciprocal off by 2 U, its product by U), the rate and its product: 7 U; the difference from zero is exact
    assert ((p.double() - want).abs() <= 7 * U * 1.01 * abs(want)).all()


@pytest.mark.parametrize("eps", [0.0, 2.0 ** -20])
def test_root_and_quotient_of_32_bit_states_are_rounded_once_each(eps):
    # beta1 = 1/2, beta2 = 0, t = 1, lr = 1/2: m = (m + g) / 2, v = g^2, the rate is one and so is the factor of the root; from p = 0 the
    # new p is the quotient itself, bit for bit the same as with numpy's float32
    n = 100_003
    g, m = normal(n, 5), normal(n, 6)
    p, v = torch.zeros(n, device="cuda"), normal(n, 7).square()
    plan = binding.AdamwPlan(ctx(), [p], [g], [binding.AdamwState(m, v)])
    a, b = g.cpu().numpy(), m.cpu().numpy()
    want_m, want_v = np.float32(0.5) * b + np.float32(0.5) * a, a * a
    binding.atomo_adamw_step(ctx(), plan, 0.5, 0.5, 0.0, eps, step=1)
    assert np.array_equal(m.cpu().numpy(), want_m) and np.array_equal(v.cpu().numpy(), want_v)
    want = -(want_m / (np.sqrt(want_v) + np.float32(eps)))
    assert want.dtype == np.float32 and np.array_equal(p.cpu().numpy(), want)
