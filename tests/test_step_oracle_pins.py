"""Pins of oracle/step_oracle.py (CPU): the definitions against autograd, torch's optimiser in float64 and hand values."""
import math

import pytest
import torch

from oracle import step_oracle as S

F64 = torch.float64


def _rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=F64)


def test_norm_of_a_constant_row_and_scale_invariance():
    x = torch.full((1, 8), 3.0, dtype=F64)
    h, rstd, y = S.rmsnorm_residual_fwd(x, None, torch.ones(8), 0.0, 1e-30)
    assert torch.allclose(y, torch.ones(1, 8, dtype=F64), atol=1e-15) and abs(float(rstd[0]) - 1 / 3) < 1e-15
    x, w = _rand(5, 33, seed=1), _rand(33, seed=2)
    _, _, a = S.rmsnorm_residual_fwd(x, None, w, 1.0, 1e-300)
    _, _, b = S.rmsnorm_residual_fwd(1024.0 * x, None, w, 1.0, 1e-300)
    assert torch.allclose(a, b, rtol=1e-14)
    assert torch.equal(S.rmsnorm_residual_fwd(x, -x, w, 0.0, 1e-6)[2], torch.zeros(5, 33, dtype=F64))


@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_norm_gradients_match_autograd(offset):
    x, r, w, dy, dh = (_rand(*s, seed=k) for k, s in enumerate([(4, 19), (4, 19), (19,), (4, 19), (4, 19)]))
    x.requires_grad_(), r.requires_grad_(), w.requires_grad_()
    h = x + r
    rstd = 1.0 / torch.sqrt((h * h).mean(1) + 1e-6)
    y = h * rstd[:, None] * (w + offset)
    ((y * dy).sum() + (h * dh).sum()).backward()
    dx, dw, _, _ = S.rmsnorm_residual_bwd(dy, dh, h, w, offset, rstd)
    assert torch.allclose(dx, x.grad, atol=1e-13) and torch.allclose(dx, r.grad, atol=1e-13)
    assert torch.allclose(dw, w.grad, atol=1e-13)


def test_norm_gradients_match_differences():
    x, w, dy = _rand(1, 7, seed=5), _rand(7, seed=6), _rand(1, 7, seed=7)
    loss = lambda x, w: float((S.rmsnorm_residual_fwd(x, None, w, 0.0, 1e-6)[2] * dy).sum())  # noqa: E731
    rstd = S.rmsnorm_residual_fwd(x, None, w, 0.0, 1e-6)[1]
    dx, dw, _, _ = S.rmsnorm_residual_bwd(dy, None, x, w, 0.0, rstd)
    e = 1e-6
    for i in range(7):
        d = torch.zeros(7, dtype=F64)
        d[i] = e
        assert abs((loss(x + d, w) - loss(x - d, w)) / (2 * e) - float(dx[0, i])) < 1e-7
        assert abs((loss(x, w + d) - loss(x, w - d)) / (2 * e) - float(dw[i])) < 1e-7


def test_adamw_matches_torch_and_the_first_step_is_a_sign():
    p0 = _rand(50, seed=3)
    p = torch.nn.Parameter(p0.clone())
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)
    q, m, v = p0.clone(), torch.zeros(50, dtype=F64), torch.zeros(50, dtype=F64)
    for t in range(1, 6):
        g = _rand(50, seed=10 + t)
        p.grad = g.clone()
        opt.step()
        q, m, v, up = S.adamw(q, g, m, v, 1e-2, 0.9, 0.999, 1e-8, 0.1, t)
        if t == 1:
            assert torch.allclose(up, torch.sign(g), atol=1e-6)
        assert torch.allclose(q, p.detach(), atol=1e-14)


def test_grad_norm_and_clip_factor():
    assert S.grad_norm([torch.tensor([3.0]), torch.tensor([4.0])], 1.0) == (5.0, 0.2)
    assert S.grad_norm([torch.tensor([0.3]), torch.tensor([0.4])], 1.0)[1] == 1.0
    assert S.grad_norm([], 1.0) == (0.0, 1.0) and S.grad_norm([torch.tensor([9.0])], 0.0) == (9.0, 1.0)


def test_e4m3_values_and_nearest_rounding_match_torch():
    vals = S.e4m3_values()
    assert torch.equal(vals.nan_to_num(nan=999.0),
                       torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).to(F64).nan_to_num(nan=999.0))
    a = torch.cat([torch.linspace(0, 448, 20001, dtype=F64), 2.0 ** torch.linspace(-14, 8.8, 20001, dtype=F64)]).float()
    got, _ = S.grid_target(a.to(F64), S.e4m3_grid(a.to(F64)), top=448.0)
    assert torch.equal(got.float(), a.to(torch.float8_e4m3fn).float())


def test_the_mean_over_all_dithers_is_the_value():
    d = torch.arange(65536)
    for a in (3.3, 0.01, 0.0007, 447.0, 17.0625):
        a16 = torch.tensor(round(a / float(S.e4m3_grid(torch.tensor(a, dtype=F64))) * 65536) / 65536
                           * float(S.e4m3_grid(torch.tensor(a, dtype=F64))), dtype=F64)
        to, _ = S.grid_target(a16.expand(65536), S.e4m3_grid(a16), d)
        assert abs(float(to.mean()) - float(a16)) < 1e-12


def test_scales_and_dithers():
    y = torch.tensor([[448.0, -1.0, 896.0, 0.0, 0.0]], dtype=F64)
    s, each = S.group_scales(y, 2)
    assert torch.equal(s, torch.tensor([[1.0, 2.0, S.SCALE_MIN]], dtype=F64)) and torch.equal(each[0, :2], torch.ones(2, dtype=F64))
    b, _ = S.block_scales(torch.cat([torch.full((256,), -448.0), torch.full((3,), 44.8)]).to(F64))
    assert torch.allclose(b, torch.tensor([1.0, 0.1], dtype=F64))
    assert S.splitmix64(0) == 0xE220A8397B1DCDAF                     # the published first outputs of seed 0
    assert S.splitmix64(0x9E3779B97F4A7C15) == 0x6E789E6AA1B965F4
    rm, rv, rp = S.dithers(4001, 7, 3, 11)
    assert all(abs(float(t.double().mean()) / 65535 - 0.5) < 0.02 and int(t.max()) < 65536 for t in (rm, rv, rp))
    assert torch.equal(S.dithers(10, 7, 3, 11)[0][2:], S.dithers(8, 7, 3, 12)[0]) and math.isfinite(float(rp.double().std()))
