"""Weight decay of the AdamW step where lr * weight_decay is near the spacing of fp32 numbers below 1 (6e-8)."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.01, 0.001])
def test_decay_adds_up_to_what_it_is_over_many_steps(bits, decay):
    """3,000 steps at lr * decay = 1e-7 and 1e-8 against the form in 64 bits: how much of theta the two differ by, as the coefficient of theta in a least-squares fit of the
    difference.  Steps of 1e-5 in random directions spread theta's roundings over its spacing, so these leave 55 * 3e-8 an element and 5e-9 in the mean of 100,000; what the
    moments' roundings and codes add has nothing to do with theta: up to 1 % of a way of 6e-4, 2e-8 in the mean.  Five times their sum is allowed, a 200th of
    the smaller sum of decays, 3e-5; a factor 1 - 1e-7 or 1 - 1e-8 in 32 bits is off by 3e-5 to 6e-5."""
    import torch
    import paper_2312_08728_amd as B
    lr, n, steps = 1e-5, 100_000, 3_000
    gen = torch.Generator(device="cuda").manual_seed(5)
    theta = torch.randn(n, generator=gen, device="cuda")
    want, m, s = theta.double(), 0.0, 0.0
    grad = torch.empty(n, device="cuda")
    opt = B.AdamW([theta], [grad], lr=lr, weight_decay=decay, state_bits=bits)
    for k in range(1, steps + 1):
        grad.normal_(generator=gen)
        opt.step()
        g = grad.double()
        m, s = 0.9 * m + 0.1 * g, 0.999 * s + 0.001 * g * g
        want = want - lr * decay * want - lr * (m / (1 - 0.9 ** k)) / ((s / (1 - 0.999 ** k)).sqrt() + 1e-8)
    off = theta.double() - want
    assert abs(float((off * want).sum() / (want * want).sum())) <= 5 * (5e-9 + 2e-8)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.0, 0.02])
def test_an_infinite_theta_stays_infinite(bits, decay):
    """theta (1 - lr decay) is the same infinity; a parameter that is one on purpose is no NaN after a step."""
    import torch
    import paper_2312_08728_amd as B
    inf = float("inf")
    theta, grad = torch.tensor([inf, -inf, 1.0], device="cuda"), torch.tensor([0.0, 1.0, 0.0], device="cuda")
    opt = B.AdamW([theta], [grad], lr=0.01, weight_decay=decay, state_bits=bits)
    for _ in range(2):
        opt.step()
    assert theta[0] == inf and theta[1] == -inf and torch.isfinite(theta[2])
