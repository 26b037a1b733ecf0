"""What rounding to 8 bits does to the moments over many steps, on the oracle (CPU).

Each seeded rounding is equal in the mean: of m, and of the root s of v.  v is the square of the stored root, so it gains
the rounding's variance at every step, E[q^2] - s^2 = f (1 - f) step^2 for a root f of a step above a code.

Bounds, derived.  Gaussian gradients of one variance, beta2 -> 1.  A root that was a code moves by Delta = s (1 - beta2) / 2 |z^2 - 1|
and its code's place by the scale's own decay, s (1 - beta2) / 2, together s (1 - beta2) / 2 z^2: f (1 - f) step^2 <= Delta step, in
the mean at most v (1 - beta2) / 2 (step / s).  step / s <= 1/8 for normal codes.  The decay of v by 1 - beta2 per step holds this at
(1/2)(1/8) = 1/16 of v at most; half that for its root is the first order, and Jensen's inequality adds the spread of v.  m: the
noise of a step is at most half a step, |m| / 16, each; it lasts 1 / (1 - beta1^2) steps."""
import pytest
import torch

from oracle import step_oracle as S

F64 = torch.float64


def settled(beta1, beta2, steps, n, seed):
    """Means over the second half of `steps` of: m8 - m, v8, v, root8, root."""
    g = torch.Generator().manual_seed(seed)
    m8 = v8 = m = v = torch.zeros(n, dtype=F64)
    sums, rms_m = torch.zeros(5, dtype=F64), 0.0
    for t in range(1, steps + 1):
        x = torch.randn(n, generator=g, dtype=F64)
        m, v = beta1 * m + (1 - beta1) * x, beta2 * v + (1 - beta2) * x * x
        kept = []
        for s in (beta1 * m8 + (1 - beta1) * x, torch.sqrt(beta2 * v8 + (1 - beta2) * x * x)):
            _, each = S.block_scales(s)
            pos = (s / each).abs()
            to, _ = S.grid_target(pos, S.e4m3_grid(pos), torch.randint(0, 65536, (n,), generator=g), top=448.0)
            kept.append(to * torch.sign(s) * each)
        root = torch.where((kept[1] == 0) & (v8 + x * x > 0), 2.0 ** -9 * each, kept[1])
        m8, v8 = kept[0], root * root
        if 2 * t > steps:
            sums += torch.stack([(m8 - m).mean(), v8.mean(), v.mean(), root.mean(), v.sqrt().mean()])
            rms_m = max(rms_m, float(m.square().mean().sqrt()))
    return sums / (steps - steps // 2), rms_m


@pytest.mark.parametrize("beta2,steps", [(0.999, 6000), (0.99, 1200), (0.95, 600)])
def test_seeded_8_bit_moments_over_many_steps(beta2, steps):
    beta1, n = 0.9, 4096
    mean, rms_m = settled(beta1, beta2, steps, n, 5)
    runs = n * (steps / 2) * (1 - beta1 ** 2)
    assert abs(float(mean[0])) <= 5 * (rms_m / 16) / (1 - beta1 ** 2) ** 0.5 / runs ** 0.5        # m: equal in the mean
    v, root = float(mean[1] / mean[2]), float(mean[3] / mean[4])
    noise = 5 * (2 * (1 - beta2) / (1 + beta2)) ** 0.5 / (n * max(1.0, steps / 2 * (1 - beta2))) ** 0.5
    assert 1.0 - noise <= v <= 1.0 + 1 / 16 + noise, v
    assert 1.0 - noise <= root <= 1.0 + 1 / 32 + noise, root
