"""Values of the layers where a formula's result is small beside what it is computed from: relative to the result itself, in 64 bits."""
import math

import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import HALF, TYPES, U, act_eval

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
