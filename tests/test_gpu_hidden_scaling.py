"""The power of two by which the gradient's coefficients are scaled while they have 16 bits: it is
that of the positions that have a gradient, whatever the others hold."""
import pytest
import torch

from test_gpu_hidden import Plain, backward, inputs

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def case(T, dtype="f16"):
    h, w, t = inputs(T, 2000, 64, dtype, seed=6, spread=0.3)
    gen = torch.Generator(device="cuda").manual_seed(T)
    g = torch.randn((T,), generator=gen, device="cuda") / T ** 2
    gh = 0.1 * torch.randn((T,), generator=gen, device="cuda") / T ** 2
    plain = Plain(h, w, t, 1.0)
    return h, w, t, g, gh, plain


def compare(got, want, tol, rows):
    assert ((got.double() - want).abs() <= tol)[rows].all()


@pytest.mark.parametrize("T", [20, 64, 400])
@pytest.mark.parametrize("value", [NAN, INF, -INF, 1e20])
def test_positions_without_a_token_left(T, value):
    """Their gradients are 0 whatever comes in for them, and the others' and the weight's as without
    them."""
    h, w, t, g, gh, plain = case(T)
    lse, H = plain.lse.float(), plain.H.float()
    lse[3], H[3] = -INF, 0.0
    gz, ghz = g.clone(), gh.clone()
    gz[3], ghz[3] = 0.0, 0.0
    dh, dw, th, tw = plain.grad(gz, ghz, "f16")
    g[3], gh[3] = value, value
    got = backward(h, w, t, 1.0, lse, H, g, gh)
    assert (got[0][3] == 0).all()
    compare(got[0], dh, th, torch.arange(T, device="cuda") != 3)
    compare(got[1], dw, tw, slice(None))


@pytest.mark.parametrize("T", [20, 64, 400])
@pytest.mark.parametrize("g3,gh3", [(NAN, 0.0), (INF, 0.0), (0.0, NAN), (-INF, INF)])
def test_a_gradient_that_is_no_number_stays_with_its_position(T, g3, gh3):
    h, w, t, g, gh, plain = case(T)
    lse, H = plain.lse.float(), plain.H.float()
    t[3] = 5
    gz, ghz = g.clone(), gh.clone()
    gz[3], ghz[3] = 0.0, 0.0
    dh, _, th, _ = plain.grad(gz, ghz, "f16")
    g[3], gh[3] = g3, gh3
    got = backward(h, w, t, 1.0, lse, H, g, gh)
    assert not got[0][3].isfinite().any() and not got[1].isfinite().any()
    compare(got[0], dh, th, torch.arange(T, device="cuda") != 3)


@pytest.mark.parametrize("T", [20, 64, 400])
@pytest.mark.parametrize("what", ["lse", "target"])
def test_a_position_without_a_distribution_stays_alone(T, what):
    """lse NaN, and a target beyond the vocabulary, beside a large gradient."""
    h, w, t, g, gh, plain = case(T)
    lse, H = plain.lse.float(), plain.H.float()
    gz, ghz = g.clone(), gh.clone()
    gz[3], ghz[3] = 0.0, 0.0
    dh, _, th, _ = plain.grad(gz, ghz, "f16")
    g[3] = 1e20
    if what == "lse":
        lse[3] = NAN
    else:
        t[3] = 2000
    got = backward(h, w, t, 1.0, lse, H, g, gh)
    assert got[0][3].isnan().all() and got[1].isnan().all()
    compare(got[0], dh, th, torch.arange(T, device="cuda") != 3)
