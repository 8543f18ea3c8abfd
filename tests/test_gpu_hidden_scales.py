"""Log-probabilities from hidden states with scales up to the largest number of fp32."""
import pytest
import torch

from test_gpu_hidden import EPS, TINY, backward, forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [3, 300])
def test_the_largest_scales(T):
    """Up to the largest number of fp32, beyond which the product with log2 e is infinite: logits of
    multiples of 2^-128, which bf16 holds."""
    V, D = 400, 16
    gen = torch.Generator(device="cuda").manual_seed(T)
    h = torch.zeros((T, D), dtype=torch.bfloat16, device="cuda")
    w = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    h[:, 0] = 2.0 ** -60
    w[:, 0] = (torch.randint(-8, 9, (V,), generator=gen, device="cuda") * 2.0 ** -66).bfloat16()
    t = torch.randint(0, V, (T,), generator=gen, device="cuda")
    for scale in (2.0 ** 126, 2.5e38, 3.4e38):
        z = scale * (h.double() @ w.double().t())
        lse = torch.logsumexp(z, 1)
        q = z - lse[:, None]
        lp, H, got = forward(h, w, t, scale)
        assert ((got.double() - lse).abs() < 1e-4).all()
        assert ((lp.double() - q.gather(1, t[:, None])[:, 0]).abs() < 1e-4).all()
        assert ((H.double() + (q * q.exp()).sum(1)).abs() < 1e-3).all()
        g = torch.randn((T,), generator=gen, device="cuda") * 2.0 ** -130
        dh, dw = backward(h, w, t, scale, got, H, g, None)
        c = -q.exp() * g.double()[:, None]
        c.scatter_add_(1, t[:, None], g.double()[:, None])
        # (c scale near 1; of what fp32 holds below 2^-126 half a step of 2^-149, then products of 2^-63)
        for a, want, size in ((dh, c @ w.double(), c.abs() @ w.double().abs()),
                              (dw, c.t() @ h.double(), c.t().abs() @ h.double().abs())):
            tol = scale * (3 * EPS["bf16"] * size + 2.0 ** -149 * 2.0 ** -60 * V)
            assert ((a.double() - scale * want).abs() <= tol + TINY["bf16"]).all()
