"""The cross entropy of a linear head at logits of any finite size, against its formulas in 64 bits.

Tolerances, u = 2^-24, r = the result type's half step.  The logits of `exact` cases are small integers or single products, which no order of the sums rounds, so that
nothing below depends on their size but where lse itself is rounded:
  lse      (3 |z - lse| + 8) u weighted with p, (32 + classes / 256) 8 u of the sums, 3 u (1 + rest) of the logarithm, rest = lse - the largest logit; and its own rounding, u |lse|
  loss     the same without lse's rounding, but with that of the difference, u |loss|
  dz       p (dloss + dlse): lse comes rounded, p = exp(z - lse) off by expm1(u |lse|) unless lse is one of fp32's values, (3 |z - lse| + 8) u; 4 u of the terms; rounded to the operands' type
  dx, dW   the terms' errors, (terms + 2) u sum |terms|, one rounding
The reference takes distances from the largest logit too: even in 64 bits 10^30 + log n is 10^30.
Other cases add e = (n + 2) u sum |terms| of the logits that are not masked (a masked one has p = 0, whatever it is)."""
import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import HALF, TYPES, U

pytestmark = pytest.mark.gpu
LOWEST = {"bf16": float(torch.finfo(torch.bfloat16).min), "f32": float(torch.finfo(torch.float32).min)}
# every tile in one piece, slices of the reduction, fp32 in three bf16 parts; and what the estimates choose
PLANS = {"bf16": ["", "product_tile=0,product_splits=1", "product_tile=1,product_splits=1", "product_tile=2,product_splits=1", "product_tile=3,product_splits=1", "product_splits=2"],
         "f32": ["", "product_tile=1,product_splits=1", "product_tile=2,product_splits=1", "product_tile=3,product_splits=1", "product_splits=2"]}
EVERY = [(dtype, plan) for dtype, plans in PLANS.items() for plan in plans]


class Case:
    """x, W, targets, and the reference from them; e: the logits' errors."""

    def __init__(self, x, w, targets, dtype, dlse=True, exact=True, masked=None, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        (rows, cin), classes = x.shape, len(w)
        self.dtype, self.x, self.w, self.targets = dtype, x.to(TYPES[dtype]), w.to(TYPES[dtype]), targets.to(torch.int32)
        self.dloss = torch.randn(rows, generator=g, device="cuda")
        self.dlse = torch.randn(rows, generator=g, device="cuda") if dlse else None
        self.z = self.x.double() @ self.w.double().t()
        self.top = self.z.max(1).values
        self.rest = (self.z - self.top[:, None]).exp().sum(1).log()
        self.lse = self.top + self.rest
        self.d = (self.z - self.top[:, None]) - self.rest[:, None]      # z - lse
        self.at = targets.long()[:, None]
        self.e = torch.zeros_like(self.z) if exact else (cin + 2) * U * (self.x.double().abs() @ self.w.double().abs().t())
        if masked is not None:
            self.e[:, masked] = 0
        self.op = B.StripeXent(rows, cin, classes, dtype)
        self.got = {n: torch.full((rows,), -7.0, device="cuda") for n in ("loss", "lse")}
        self.dx, self.dw = torch.full_like(self.x, -7.0), torch.full_like(self.w, -7.0)

    def forward(self):
        self.op.run(self.x, self.w, self.targets, self.got["loss"], self.got["lse"])

    def backward(self, lse):
        self.op.backward(self.x, self.w, self.targets, lse, dloss=self.dloss, dlse=self.dlse, dx=self.dx, dw=self.dw)

    def check_forward(self):
        d, lse = self.d, self.lse
        tol = self.e.max(1).values + (d.exp() * (3 * d.abs().clamp(max=1e4) + 8) * U).sum(1) + (32 + d.shape[1] / 256) * 8 * U + 3 * U * (1 + self.rest)
        want = -d.gather(1, self.at)[:, 0]
        off = (self.got["loss"].double() - want).abs()
        tolerance = tol + self.e.gather(1, self.at)[:, 0] + U * want.abs()
        assert (off <= tolerance).all(), f"loss: {float((off / tolerance).max()):.3g} of the tolerance"
        off, tolerance = (self.got["lse"].double() - lse).abs(), tol + U * lse.abs()
        assert (off <= tolerance).all(), f"lse: {float((off / tolerance).max()):.3g} of the tolerance"

    def check_backward(self, lse_exact=False):
        r, x, w = HALF[self.dtype], self.x.double(), self.w.double()
        lse_off = 0.0 if lse_exact else U * self.lse.abs()[:, None]
        one = self.dloss.double()
        both = one + self.dlse.double() if self.dlse is not None else one
        p = self.d.exp()
        dz = p * both[:, None]
        dz.scatter_add_(1, self.at, -one[:, None])
        size = p * both.abs()[:, None]
        size.scatter_add_(1, self.at, one.abs()[:, None])
        d = self.d.abs().clamp(max=1e4)
        dzt = p * both.abs()[:, None] * (torch.expm1(self.e + lse_off) + 3 * U * d + 8 * U) + 4 * U * size
        dzt = dzt + r * (dz.abs() + dzt)
        for name, got, want, tol in (("dx", self.dx, dz @ w, (dzt + (len(w) + 3) * U * dz.abs()) @ w.abs()),
                                     ("dw", self.dw, dz.t() @ x, (dzt + (len(x) + 2) * U * dz.abs()).t() @ x.abs())):
            tol = (tol + r * want.abs()) * (1 + r) + 1e-35
            off = (got.double() - want).abs()
            assert (off <= tol).all(), f"{name}: {int((~(off <= tol)).sum())} of {off.numel()} off, worst {float((off / tol).max()):.3g} of the tolerance"


def sure(rows, classes, cin, dtype, power, seed=0):
    """Rows whose largest logit is some 10^power, far above all others: one class's weights are 1, those of the others -1."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, w = torch.zeros(rows, cin, device="cuda"), torch.zeros(classes, cin, device="cuda")
    x[:, 0] = (10.0 ** power * (1 + torch.rand(rows, generator=g, dtype=torch.float64, device="cuda"))).to(TYPES[dtype]).float()
    w[:, 0] = -1
    w[classes // 3, 0] = 1
    targets = torch.where(torch.arange(rows, device="cuda") % 2 == 0, classes // 3, (torch.arange(rows, device="cuda") * 7) % classes)
    return x, w, targets


@pytest.mark.parametrize("power", [4, 5, 6, 7, 8, 9, 12, 20, 30, 38])
@pytest.mark.parametrize("dtype,plan", EVERY)
def test_loss_of_sure_rows(monkeypatch, dtype, plan, power):
    """lse is the largest logit itself, the loss 0, or the distance of two logits: nothing in them is rounded."""
    monkeypatch.setenv("STRIPE_TUNE", plan)
    t = Case(*sure(70, 700, 520, dtype, power), dtype)
    t.forward()
    top = t.x[:, 0].float()
    assert torch.equal(t.got["lse"], top)
    assert torch.equal(t.got["loss"], torch.where(t.targets == 700 // 3, torch.zeros_like(top), 2 * top))


@pytest.mark.parametrize("power", [4, 5, 6, 7, 8, 9, 12, 20, 30])
@pytest.mark.parametrize("dtype,plan", EVERY)
def test_gradients_of_sure_rows(monkeypatch, dtype, plan, power):
    """p is 1 for the largest logit and 0 for all others: dz is made of the weights alone."""
    monkeypatch.setenv("STRIPE_TUNE", plan)
    t = Case(*sure(70, 700, 520, dtype, power), dtype)
    t.backward(t.x[:, 0].float().contiguous())
    t.check_backward(lse_exact=True)


@pytest.mark.parametrize("dtype,plan", EVERY)
def test_gradients_never_pass_their_weights(monkeypatch, dtype, plan):
    """Logits of some 1e9 whose last bits are worth 64, added up in one order for lse and in another for dz: still 0 <= p <= 1, so |dz| <= |dloss| + |dlse|."""
    monkeypatch.setenv("STRIPE_TUNE", "product_splits=2" if "splits=2" not in plan else "product_tile=2,product_splits=1")
    g = torch.Generator(device="cuda").manual_seed(5)
    rows, classes, cin = 130, 600, 520
    args = (torch.randn(rows, cin, generator=g, device="cuda") * 1e4, torch.randn(classes, cin, generator=g, device="cuda") * 1e4, torch.arange(rows, device="cuda") * 3, dtype)
    first = Case(*args, exact=False)
    first.forward()
    monkeypatch.setenv("STRIPE_TUNE", plan)
    t = Case(*args, exact=False)
    t.backward(first.got["lse"])
    weight = t.dloss.abs().double() + t.dlse.abs().double()
    more = 1 + 2 * HALF[dtype] + (classes + 8) * U      # dz's rounding and the result's, the sums'
    assert (t.dw.double().abs() <= weight @ t.x.double().abs() * more).all()
    assert (t.dx.double().abs() <= (weight[:, None] * t.w.double().abs().sum(0)) * more).all()


@pytest.mark.parametrize("dtype,plan", EVERY)
def test_loss_between_logits_near_one_another(monkeypatch, dtype, plan):
    """Integers around 2^20, 2^23 and -2^22: what the loss is made of is some units in size."""
    monkeypatch.setenv("STRIPE_TUNE", plan)
    rows, classes, cin = 90, 600, 520
    x, w = torch.zeros(rows, cin, device="cuda"), torch.zeros(classes, cin, device="cuda")
    x[:, 0] = torch.tensor([2.0 ** 20, 2.0 ** 23, -2.0 ** 22], device="cuda").repeat(rows // 3)
    x[:, 1] = 1
    w[:, 0], w[:, 1] = 1, -(torch.arange(classes, device="cuda") * 37 % 23).float()
    t = Case(x, w, torch.arange(rows, device="cuda") * 5 % classes, dtype)
    t.forward()
    t.check_forward()


MASKS = [-1e5, -1e10, -1e30, None]      # None: the type's lowest value


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype,plan", EVERY)
@pytest.mark.parametrize("rows", [5, 150])
def test_loss_with_finite_masks(monkeypatch, dtype, plan, mask, rows):
    """Classes that a large negative weight masks: one here and there, all that a wavefront has, whole tiles."""
    monkeypatch.setenv("STRIPE_TUNE", plan)
    t = with_masks(rows, dtype, mask)
    t.forward()
    t.check_forward()


def with_masks(rows, dtype, mask):
    g = torch.Generator(device="cuda").manual_seed(rows)
    classes, cin = 1300, 520
    x, w = torch.randn(rows, cin, generator=g, device="cuda"), torch.randn(classes, cin, generator=g, device="cuda") * cin ** -0.5
    masked = torch.zeros(classes, dtype=torch.bool, device="cuda")
    masked[512:1024] = True
    masked[64:160] = True
    masked[1::5] = True
    x[:, 3] = 1
    w[:, 3] = torch.where(masked, LOWEST[dtype] if mask is None else mask, 0.0)
    open_classes = torch.arange(classes, device="cuda")[~masked]
    targets = open_classes[torch.randint(0, len(open_classes), (rows,), generator=g, device="cuda")]
    return Case(x, w, targets, dtype, exact=False, masked=masked)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype,plan", EVERY)
def test_gradients_with_finite_masks(monkeypatch, dtype, plan, mask):
    monkeypatch.setenv("STRIPE_TUNE", plan)
    t = with_masks(150, dtype, mask)
    t.backward(t.lse.float())
    t.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_of_rows_that_are_masked_altogether(dtype):
    """Every logit is the same large negative number: the loss is the logarithm of the classes' number."""
    rows, classes, cin = 20, 300, 64
    for value in (-1e6, -1e30, LOWEST[dtype]):
        x, w = torch.zeros(rows, cin, device="cuda"), torch.zeros(classes, cin, device="cuda")
        x[:, 5], w[:, 5] = 1, value
        t = Case(x, w, torch.arange(rows, device="cuda"), dtype)
        t.forward()
        t.check_forward()


@pytest.mark.parametrize("rows", [7, 64, 65])
@pytest.mark.parametrize("cin", [520, 333])
@pytest.mark.parametrize("dtype,plan", EVERY)
def test_rows_that_do_not_count_reach_no_other(monkeypatch, dtype, plan, cin, rows):
    """The same bits for the rows that count, whatever the others hold: few rows are read where they lie."""
    monkeypatch.setenv("STRIPE_TUNE", plan)
    g = torch.Generator(device="cuda").manual_seed(cin + rows)
    x, w = torch.randn(rows, cin, generator=g, device="cuda"), torch.randn(700, cin, generator=g, device="cuda")
    targets = torch.arange(rows, device="cuda") * 5
    t = Case(x, w, targets, dtype, exact=False)
    ignored = torch.arange(rows, device="cuda") % 3 == 1
    t.targets[ignored] = -1
    results = []
    for value in (0.0, float("nan"), float("inf"), 3e38):
        t.x[ignored] = value
        t.forward()
        assert (t.got["loss"][ignored] == 0).all() and (t.got["lse"][ignored] == 0).all()
        lse = t.lse.float()
        lse[ignored] = t.dloss[ignored] = t.dlse[ignored] = value
        t.backward(lse)
        assert (t.dx[ignored] == 0).all()
        results.append(torch.cat([t.got["loss"][~ignored], t.got["lse"][~ignored], t.dx.float().flatten(), t.dw.float().flatten()]))
    assert torch.isfinite(results[0]).all() and all(torch.equal(results[0], r) for r in results)
