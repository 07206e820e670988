"""Layer norm of rows whose mean is far larger than their spread."""
import pytest
import torch

from tests import train_ref as R

pytestmark = pytest.mark.gpu
KINDS = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def G():
    from paper_2402_09633_amd import gnn
    return gnn


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("k", [1, 7, 96, 128, 391, 1000, 2048, 2056, 8192, 16_383])
def test_constant_rows(G, k, kind):
    """Their mean is the number itself, and what they deviate by is nothing."""
    c = torch.tensor([0.1, -1000.1, 3000.1, 59_999.0, 1e-5, 0.0, -0.3], device="cuda").to(KINDS[kind])
    x = c[:, None].expand(7, k).contiguous()
    g = torch.Generator(device="cuda").manual_seed(k)
    gamma = 1 + 0.2 * torch.randn(k, device="cuda", generator=g)
    beta = 0.1 * torch.randn(k, device="cuda", generator=g)
    dy = torch.randn(7, k, device="cuda", generator=g).to(KINDS[kind])
    eps = 1e-5
    y, mean, rstd = G.layer_norm(x, gamma, beta, eps, save=True)
    assert torch.equal(y, beta.to(y.dtype).expand(7, -1))
    assert torch.equal(mean, c.float())
    # The squares of deviations by d and the square of their mean, both d^2, differ by
    # their sums' roundings, some 100 U d^2; |d| itself is at most 48 U |c|, so that
    # 100 U (48 U 6e4)^2 = 2e-7 stays of eps at most, half of that in rstd.
    assert ((rstd.double() * eps ** 0.5 - 1).abs() <= 0.5 * 2e-7 / eps + 4 * R.U).all()
    for have, (v, e) in zip(G.layer_norm_backward(dy, x, gamma, mean, rstd),
                            R.layer_norm_backward(dy, x, gamma, eps)):
        R.within(have, v, e)


@pytest.mark.parametrize("k", [64, 300, 2500])
def test_the_mean_is_right_to_its_last_place(G, k):
    g = torch.Generator(device="cuda").manual_seed(k)
    x = 3000.1 + torch.randn(200, k, device="cuda", generator=g)
    one, zero = torch.ones(k, device="cuda"), torch.zeros(k, device="cuda")
    y, mean, rstd = G.layer_norm(x, one, zero, save=True)
    want = x.double().mean(1)
    # half a place, and what the deviations' own mean (below 48 U |mean| of them, plus
    # their spread's roundings) leaves
    assert ((mean.double() - want).abs() <= 1.01 * R.U * want.abs() + 50 * R.U * 4.0).all()
    d = x.double() - want[:, None]
    r = 1 / ((d * d).mean(1, keepdim=True) + 1e-5).sqrt()
    # the common shift by a rounded mean, two roundings of each deviation, the variance
    # (50 roundings and the shift's square), the product
    bound = r * (1.01 * R.U * want.abs()[:, None] + 200 * R.U) + (d * r).abs() * 40 * R.U
    R.within(y, d * r, bound)
