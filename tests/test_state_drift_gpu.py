"""The update's 8-bit states against its float32 states over many steps on the same gradients.

The bounds are those of test_state_drift_cpu.py: m is equal in the mean (5 standard deviations of its rounding noise), v is above
the float32 v by 1/16 of itself at most, its root by 1/32, and by 5 standard deviations of the two averages."""
import pytest
import torch

from paper_2605_07244_b200 import binding as B
from paper_2605_07244_b200 import build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beta2,steps", [(0.999, 5000), (0.95, 600)])
def test_seeded_states_settle_where_the_oracle_says(beta2, steps):
    build.build()
    beta1, n = 0.9, 1 << 16
    g = torch.Generator(device="cuda").manual_seed(3)
    grad = torch.empty(n, device="cuda")
    f = lambda k=n: torch.zeros(k, device="cuda")  # noqa: E731
    m, v, ms, vs = f(), f(), f(n // B.STATE_BLOCK), f(n // B.STATE_BLOCK)
    m8, v8 = (torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
    tensors = B.TensorList([B.TensorSlot(grad, f(), None, m, v), B.TensorSlot(grad, f(), None, m8, v8, ms, vs, rng_first=7)])
    ap = B.AdamwParams(lr=1e-6, beta1=beta1, beta2=beta2, eps=1e-8, seed=11, rounding=B.ROUND_SEEDED)
    sums, rms_m = torch.zeros(5, dtype=torch.float64, device="cuda"), 0.0
    wide = lambda q, s: (q.float().view(-1, B.STATE_BLOCK) * s[:, None]).view(-1).double()  # noqa: E731
    for t in range(1, steps + 1):
        grad.normal_(generator=g)
        ap.step = t
        B.mrl_adamw_step(tensors, ap)
        if 2 * t > steps:
            root = wide(v8, vs)
            sums += torch.stack([(wide(m8, ms) - m.double()).mean(), root.square().mean(), v.double().mean(), root.mean(),
                                 v.double().sqrt().mean()])
    rms_m = float(m.double().square().mean().sqrt())
    mean = (sums / (steps - steps // 2)).cpu()
    runs = n * (steps / 2) * (1 - beta1 ** 2)
    assert abs(float(mean[0])) <= 5 * (rms_m / 16) / (1 - beta1 ** 2) ** 0.5 / runs ** 0.5
    at_v, at_root = float(mean[1] / mean[2]), float(mean[3] / mean[4])
    noise = 5 * (2 * (1 - beta2) / (1 + beta2)) ** 0.5 / (n * max(1.0, steps / 2 * (1 - beta2))) ** 0.5
    assert 1.0 - noise <= at_v <= 1.0 + 1 / 16 + noise and 1.0 - noise <= at_root <= 1.0 + 1 / 32 + noise, (at_v, at_root)
