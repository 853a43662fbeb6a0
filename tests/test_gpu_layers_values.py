"""Values of the layers where a formula's result is small beside what it is computed from: relative to the result itself, in 64 bits."""
import math

import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import HALF, TYPES, U, Norm, act_eval

pytestmark = pytest.mark.gpu


def column(z, dtype, act, rows):
    """act(z) and act'(z) for a column of values, by a layer whose x is (1, 0, 0, ...) and whose weights are z in their first column."""
    n, cin = z.numel(), 8
    x, w = torch.zeros(rows, cin, dtype=z.dtype, device="cuda"), torch.zeros(n, cin, dtype=z.dtype, device="cuda")
    x[:, 0], w[:, 0] = 1.0, z
    y, db = torch.full((rows, n), -7.0, dtype=z.dtype, device="cuda"), torch.full((n,), -7.0, device="cuda")
    B.StripeLinear(rows, cin, n, dtype, activation=act).run(x, w, y)
    B.StripeLinear(1, cin, n, dtype, activation=act).backward(torch.ones_like(z)[None], x[:1], w, pre=z[None], dbias=db)
    torch.cuda.synchronize()
    return y, db


@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_activations_of_negative_values(act, dtype, rows):
    """Down to where results leave fp32's range, with a tolerance relative to the result.

    act_eval bounds the evaluation's relative error (the exponent's argument, exp, erfc, the quotient); bf16 gelu takes the normal distribution
    function from a polynomial, at most 2^-14 of it off.  Results below 2^-118 in size may be 0.  act'(z) = Phi + z phi and the like
    cancel: relative to the sum of its terms' sizes, two fp32 roundings more."""
    if dtype == "bf16":
        low = {"gelu": -13.25, "gelu_tanh": -10.5, "silu": -90.0}[act]
        z = torch.arange(0x3a80, 0x4300, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16)       # every value from 2^-10 to 128
        z = -z[z.float() <= -low]
    else:
        z = torch.linspace({"gelu": -13.2, "gelu_tanh": -10.4, "silu": -90.0}[act], 0, 4001, device="cuda")
    zd = z.double()
    if act == "gelu_tanh":       # z / 2 (1 + tanh(u)) = z / (1 + exp(-2u)), which does not cancel in 64 bits
        u2 = 2 * math.sqrt(2 / math.pi) * (zd + 0.044715 * zd ** 3)
        p = torch.sigmoid(u2)
        want, second = zd * p, zd * p * (1 - p) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * zd * zd)
    elif act == "gelu":
        p = torch.special.erfc(-zd / math.sqrt(2)) / 2       # (ndtr is 0 below -8.4)
        want = zd * p
        second = zd * torch.exp(-zd * zd / 2) / math.sqrt(2 * math.pi)
    else:
        p = torch.sigmoid(zd)
        want, second = zd * p, zd * p * (1 - p)
    slope = p + second
    rel = act_eval(zd, act) + (2.0 ** -14 if dtype == "bf16" and act == "gelu" else 0)
    y, db = column(z, dtype, act, rows)
    tol = rel * want.abs()
    tol = tol + HALF[dtype] * (want.abs() + tol) + 2.0 ** -118
    err = ((y.double() - want).abs() / tol).max(0).values
    assert err.max() <= 1, f"act({z[err.argmax()].item()}): {y[0, err.argmax()].item()} for {want[err.argmax()].item()}, {err.max().item():.2f} of the tolerance"
    tol = (rel + 6 * U) * (p + second.abs()) + 2.0 ** -118
    err = (db.double() - slope).abs() / tol
    assert err.max() <= 1, f"act'({z[err.argmax()].item()}): {db[err.argmax()].item()} for {slope[err.argmax()].item()}, {err.max().item():.2f} of the tolerance"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("features", [7, 64, 1000, 3001, 8192, 16384, 16391, 40000])
def test_norm_of_constant_rows(features, dtype):
    """h = 0, y = beta and mean = x, whatever x is.

    n fp32 additions after one another leave a first mean m that is off by d, |d| <= n u |x|; the distances from it are exact and all d, their mean is d
    up to n u |d|: h is off by (n u)^2 |x| / sqrt(eps), and the mean by that and its own rounding."""
    value = torch.tensor([0.1, 1000.1, -77777.7, 3e-3, 0.0], device="cuda").to(TYPES[dtype])
    x = value[:, None].expand(-1, features).contiguous()
    rows, eps, n = len(value), 1e-5, 32 + 6 + 16 + features // 1024 + 4
    g = torch.Generator(device="cuda").manual_seed(features)
    gamma, beta = (torch.randn(features, generator=g, device="cuda") for _ in range(2))
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.StripeNorm(rows, features, dtype, eps=eps).run(x, y, gamma=gamma, beta=beta, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    v = value.double()
    left = (n * U) ** 2 * v.abs()
    assert ((mean.double() - v).abs() <= left + U * (v.abs() + left)).all(), (mean, value)
    tol = left[:, None] * eps ** -0.5 * gamma.double().abs() + U * beta.double().abs()
    err = (y.double() - beta.double()).abs()
    tol = tol + HALF[dtype] * (beta.double().abs() + tol)
    assert (err <= tol).all(), [(value[r].item(), err[r].max().item(), tol[r].max().item()) for r in range(rows)]
    # var <= (n u x)^2 changes eps by that much
    s = eps ** -0.5
    assert ((rstd.double() - s).abs() <= s * ((n * U * v) ** 2 / eps + 6 * U)).all(), rstd


def test_norm_of_rows_whose_mean_is_far_larger_than_their_spread():
    """x = m (1 + k 2^-20), |k| <= 3: the spread is a few of fp32's steps.  The first mean is off by up to n u |m|, more than the spread; the corrected
    one by (n u)^2 |m| + n u mean |x - m| and its own rounding."""
    rows, features, n = 40, 3001, 32 + 6 + 16 + 8
    g = torch.Generator(device="cuda").manual_seed(7)
    m = 2.0 ** torch.randint(-3, 12, (rows, 1), generator=g, device="cuda").float()
    x = m * (1 + torch.randint(-3, 4, (rows, features), generator=g, device="cuda").float() * 2.0 ** -20)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    eps = 1e-12
    B.StripeNorm(rows, features, "f32", eps=eps).run(x, y, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    xd = x.double()
    mu = xd.mean(1, keepdim=True)
    d = xd - mu
    var = (d * d).mean(1, keepdim=True) + eps
    s = var ** -0.5
    # distances from the first mean are at most |d| + n u |m|, which their squares' sum and the correction's square carry into the variance
    wide = d.abs() + n * U * xd.abs()
    em = (n * U) ** 2 * xd.abs().mean(1, keepdim=True) + (n + 2) * U * wide.mean(1, keepdim=True)
    es = s * ((n + 8) * U * 2 * (wide * wide).mean(1, keepdim=True) / var + em * em / var + 8 * U)
    ey = (em + U * mu.abs() + 2 * U * wide) * s + d.abs() * es + 3 * U * (d * s).abs()
    assert ((mean.double()[:, None] - mu).abs() <= em + U * mu.abs()).all()
    assert ((rstd.double()[:, None] - s).abs() <= es + U * s).all()
    assert ((y.double() - d * s).abs() <= ey).all(), ((y.double() - d * s).abs() / ey).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("features", [7, 3001, 16384, 40000])
def test_norm_of_rows_with_infinities_nan_and_large_values(features, dtype):
    """An infinity in a row is its mean and leaves no finite distance; equal values whose distances from a rounded mean have no finite square are beta still."""
    x = torch.randn(6, features, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda").to(TYPES[dtype])
    x[0, 3], x[1, features - 1], x[2, 1], x[3], x[4] = float("inf"), float("-inf"), float("nan"), 1e30, -1e26
    beta = torch.randn(features, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    B.StripeNorm(6, features, dtype).run(x, y, beta=beta, mean=mean, rstd=rstd)
    torch.cuda.synchronize()
    assert mean[0] == float("inf") and mean[1] == float("-inf") and torch.isnan(mean[2]) and torch.isnan(rstd[:3]).all() and torch.isnan(y[:3]).all()
    n = 32 + 6 + 16 + features // 1024 + 4
    assert ((mean[3:5].double() - x[3:5, 0].double()).abs() <= n * U * x[3:5, 0].double().abs()).all()
    # the mean is exact, or its error's square overflows and s is 0
    assert torch.equal(y[3:5], beta.to(y.dtype).expand(2, -1))
    assert torch.isfinite(y[5]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,features", [(300, 20000), (1100, 16392), (77, 131075), (9, (1 << 21) + 1)])
def test_norm_of_long_rows(rows, features, dtype):
    """Column sums in one, a few and many workgroups to a strip of columns."""
    c = Norm(rows, features, dtype)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("other", [2.0 ** 40, 2.0 ** 60])
@pytest.mark.parametrize("splits", [1, 3])
def test_f32_in_parts_of_small_values(splits, other, monkeypatch):
    """Three bf16 parts hold all 24 bits of a value down to 2^-110, and of a smaller one what does not lie below 2^-133.

    One value in each row: the result is a single product, six products of parts added up with a rounding or truncation each, at most 2 u, and the dropped
    ones below 2^-25 of it: within 14 u.  A part that ends at 2^-133 is off by half of that, times the other factor."""
    monkeypatch.setenv("STRIPE_TUNE", f"product_few=0,product_tile=1,product_splits={splits}")
    rows, cin, cout = 200, 421, 389
    op = B.StripeLinear(rows, cin, cout, "f32")
    name = "_parts" + (f"_k{splits}" if splits > 1 else "")
    assert all(op.info[k].endswith(name) for k in ("forward", "input_grad", "weight_grad")), op.info
    g = torch.Generator(device="cuda").manual_seed(1)

    def single(n, m, exponent):       # a value from 2^exponent to twice that in each row of a matrix, of either sign
        v = torch.zeros(n, m, dtype=torch.float64, device="cuda")
        size = (1 + torch.rand(n, generator=g, device="cuda", dtype=torch.float64)) * 2.0 ** exponent
        v[torch.arange(n, device="cuda"), torch.randint(0, m, (n,), generator=g, device="cuda")] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, size, -size)
        return v.float()

    def dense(n, m):
        return (1 + torch.rand(n, m, generator=g, device="cuda")) * other

    for exponent in (0, -60, -100, -109, -110, -111, -118, -125, -130, -133, -140):
        for first in (True, False):       # the small values in the first operand, in the second
            x, w, dy = (single(rows, cin, exponent), dense(cout, cin), single(rows, cout, exponent)) if first else (
                dense(rows, cin), single(cout, cin, exponent), dense(rows, cout))
            wt = w if first else single(cin, cout, exponent).t().contiguous()      # dx: one value in each column of W
            xs, dys = (single(cin, rows, exponent).t().contiguous(), dense(rows, cout)) if first else (dense(rows, cin), single(cout, rows, exponent).t().contiguous())
            y, dx, dw = torch.empty(rows, cout, device="cuda"), torch.empty_like(x), torch.empty_like(w)
            op.run(x, w, y)
            op.backward(dy, x, wt, dx=dx)
            op.backward(dys, xs, w, dw=dw)
            torch.cuda.synchronize()
            for what, got, a, b in (("y", y, x, w.t()), ("dx", dx, dy, wt), ("dw", dw, dys.t(), xs)):
                v = a.double() @ b.double()
                tol = 14 * U * v.abs() + (2.0 ** -134 * 2 * other if exponent < -110 else 0)
                worst = (got.double() - v).abs() / tol
                assert (worst <= 1).all(), f"{what}: {worst.max().item():.1f} of the tolerance, values from 2^{exponent}"
