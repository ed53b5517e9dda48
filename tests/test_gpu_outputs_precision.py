"""How many digits the operators beside the decoder keep where a value is small: against the definitions in 64 bits, relative to the
value itself.

u = 2^-24 is half a step of fp32.  The hardware's 2^x and 1 / x are within a step (2u), everything else rounds once (u)."""
import math

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2311_04996_amd import linear, token_logprobs, token_logprobs_backward  # noqa: E402

U = 2.0 ** -24
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def relative(got, want, tol, dtype=torch.float32):
    """got within tol of want, relative to it, and the rounding to a 16-bit result."""
    want = want.double()
    if dtype != torch.float32:
        f = torch.finfo(dtype)
        tol = want.abs() * (tol + f.eps / 2) + f.smallest_normal * f.eps / 2
    else:
        tol = want.abs() * tol
    off = ((got.double() - want).abs() - tol)
    assert float(off.max()) <= 0, f"off by {float(((got.double() - want).abs() / want.abs().clamp(min=1e-300)).max()) / U:.1f} u"


def through(z, n, act, out):
    """act of the column z by way of linear: z times 1 is z itself, in every one of n columns."""
    got = linear(z[:, None], torch.ones((n, 1), dtype=z.dtype, device="cuda"), activation=act, out_dtype=DT[out])
    assert bool(((got == got[:, :1]) | torch.isnan(got)).all())
    return got[:, 0]


# rows and columns: 16 x 16, 32 x 64 or 64 x 64 and larger tiles
@pytest.mark.parametrize("m,n", [(4001, 1), (40001, 1), (9001, 130)])
@pytest.mark.parametrize("out", DT)
def test_gelu_keeps_its_digits(m, n, out):
    """fp32: t 3u (a sum and the hardware's 1 / x), and F goes like t at most: 3u; its coefficients, roundings and fit 4u; e^d 3u;
    two products 2u: 12u.  Below 1: three roundings of erf <= 0.68 and one of 1 - erf >= 0.32: 8u, and the product.  16 bits: the fit
    36u, and the exponent d <= 72 is off by 2.25 u d."""
    z = torch.linspace(-12, 9, m, device="cuda")
    want = z.double() * 0.5 * torch.special.erfc(-z.double() / math.sqrt(2.0))
    relative(through(z, n, "gelu", out), want, 14 * U if out == "f32" else 256 * U, DT[out])
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e4, -1e4, 3e38, -3e38, math.inf, math.nan], device="cuda")
    got = through(z, n, "gelu", "f32").tolist()
    assert got[:2] == [0, 0] and got[4] == 1e4 and got[5] == 0 and got[7] == 0 and got[8] == math.inf and math.isnan(got[9])
    assert abs(got[2] / 1e-30 - 0.5) < 1e-6 and abs(got[3] / 1e-30 + 0.5) < 1e-6 and abs(got[6] / 3e38 - 1) < 1e-6


@pytest.mark.parametrize("m,n", [(4001, 1), (40001, 1), (9001, 130)])
@pytest.mark.parametrize("out", DT)
def test_silu_keeps_its_digits(m, n, out):
    """fp32: e^-z 3u (the hardware's 2^x, and what the exponent lost put back), the sum and the quotient u each.  16 bits: the exponent is off
    by 1.25 u |z|, and 1 / x and a product come to it."""
    z = torch.linspace(-80, 20, m, device="cuda")
    relative(through(z, n, "silu", out), z.double() * torch.sigmoid(z.double()), 7 * U if out == "f32" else 128 * U, DT[out])
    z = torch.tensor([0.0, -0.0, 1e-30, 1e4, -1e4, 3e38, -3e38, math.inf, math.nan, -88.5], device="cuda")
    got = through(z, n, "silu", "f32").tolist()
    assert got[:2] == [0, 0] and abs(got[2] / 5e-31 - 1) < 1e-6 and got[3] == 1e4 and got[4] == 0 and got[6] == 0 and got[7] == math.inf
    assert abs(got[5] / 3e38 - 1) < 1e-6 and math.isnan(got[8]) and abs(got[9] / (-88.5 * math.exp(-88.5)) - 1) < 1e-5


@pytest.mark.parametrize("v", [29, 129, 500, 2048, 2049, 40001])
def test_the_gradient_keeps_the_digits_of_small_probabilities(v):
    """The gradient of lse is p itself, e^(x - maximum - log_sum) of the forward call's maximum and log_sum.  The roundings of the two
    differences are kept: the hardware's 2^x 2u, what is put back u, the product with the slope of 1 nothing: 3u, and 2^-24 of
    the roundings themselves."""
    g = torch.Generator(device="cuda").manual_seed(v)
    x = torch.randn((50, v), generator=g, device="cuda") * 6
    x[:, 0] = torch.linspace(-60, 0, 50, device="cuda")
    r = token_logprobs(x)
    want = torch.exp((x.double() - r.maximum.double()[:, None]) - r.log_sum.double()[:, None])
    got = token_logprobs_backward(x, r, grad_lse=torch.ones(50, device="cuda"))
    assert float(want.min()) >= 2.0 ** -126                                        # (all of them normal numbers)
    relative(got, want, 5 * U)
