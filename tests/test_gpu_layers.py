"""The layers (linear layer with its epilogue, rows sorted by expert, layer norm; forward and gradients) on the GPU against their
formulas in 64 bits.

Tolerances, u = 2^-24, r = the result type's half step (bf16 2^-8, fp32 2^-24), derived per element:
  sums     n terms added in any order in fp32: n u sum |terms| (a product entering a matrix instruction is exact or rounded once more,
           which the n leaves room for: n + 2)
  act(z)   |act'| <= 1.13, so an error e of z becomes at most 1.13 e; evaluating act itself: the exponent's argument a is rounded a few
           times, |a| <= 2 (|z| + 0.045 |z|^3), which makes exp, erfc and the quotient off by (4 |a| + z^2 + 16) 2 u relative to |z|
  act'(z)  the same relative to 1 + |z|
  dz       is rounded to the operands' type before the two products: r |dz| into each term
  result   one rounding, r |result|
"""
import math

import numpy as np
import pytest
import torch

from paper_1903_06498_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
U = 2.0 ** -24
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
NAN = float("nan")


def act_ref(z, name):
    """act(z), act'(z) in 64 bits."""
    if name == "relu":
        return z.clamp(min=0), (z > 0).double()
    if name == "gelu":
        p = torch.special.ndtr(z)
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = torch.tanh(a * (z + 0.044715 * z ** 3))
        return z * (1 + t) / 2, (1 + t) / 2 + z / 2 * (1 - t * t) * a * (1 + 0.134145 * z * z)
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def act_eval(z, name):
    """Relative error of evaluating act or act' in fp32 (see above)."""
    z = z.abs()
    return 0 * z if name in ("none", "relu") else (8 * (z + 0.045 * z ** 3) + z * z + 16) * 2 * U


def window(shape, row, dtype, offset=0, fill=NAN):
    """A [..., n] window with rows `row` apart whose first element lies `offset` elements into its buffer, everything around it `fill`."""
    n_rows = int(np.prod(shape[:-1]))
    buf = torch.full((offset + n_rows * row + 64,), fill, dtype=dtype, device="cuda")
    strides = [1, row]
    for d in reversed(shape[1:-1]):
        strides.append(strides[-1] * d)
    return buf, torch.as_strided(buf, shape, list(reversed(strides)), offset)


def untouched(buf, view, fill):
    """Whether the buffer holds `fill` wherever `view` does not reach."""
    seen = torch.zeros_like(buf, dtype=torch.bool)
    torch.as_strided(seen, view.shape, view.stride(), view.storage_offset()).fill_(True)
    rest = buf[~seen]
    return bool((torch.isnan(rest) if fill != fill else rest == fill).all())


def bounds(offsets, rows):
    """Rows of each group as the library reads them: running maximum, limited to the rows."""
    ends = np.maximum.accumulate(np.clip(np.array(offsets, dtype=np.int64), 0, rows))
    return list(zip(ends[:-1].tolist(), ends[1:].tolist()))


class Linear:
    """Inputs of one layer, the library's results, the formulas' values and the tolerances."""

    def __init__(self, rows, cin, cout, dtype, act="none", offsets=None, bias=True, residual=True, pad=0, shift=0, seed=0, scale=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt, self.dtype, self.act, self.rows = TYPES[dtype], dtype, act, rows
        groups = len(offsets) - 1 if offsets is not None else 0
        lead = (groups,) if groups else ()

        def make(*shape, s=1.0):
            buf, v = window(shape, shape[-1] + pad, dt, shift)
            v.copy_((torch.randn(*shape, generator=g, device="cuda") * s).to(dt))
            return v

        self.x, self.w = make(rows, cin, s=scale), make(*lead, cout, cin, s=cin ** -0.5)
        self.dy, self.pre_in = make(rows, cout), make(rows, cout, s=1.5)
        self.residual = make(rows, cout) if residual else None
        self.bias = torch.randn(*lead, cout, generator=g, device="cuda") if bias else None
        self.offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda") if groups else None
        self.spans = bounds(offsets, rows) if groups else [(0, rows)]
        self.inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
        for a, b in self.spans:
            self.inside[a:b] = True
        for t in (self.x, self.dy, self.pre_in):
            t[~self.inside] = NAN                      # rows of no group are read by nobody
        if residual:
            self.residual[~self.inside] = NAN
        self.outs = {}
        for name, shape in (("y", (rows, cout)), ("pre", (rows, cout)), ("dx", (rows, cin)), ("dw", lead + (cout, cin))):
            self.outs[name] = window(shape, shape[-1] + pad, dt, shift, -7.0)
        self.dbias = torch.full(lead + (cout,), -7.0, device="cuda")
        self.op = B.StripeLinear(rows, cin, cout, dtype, activation=act, groups=groups, x_row=cin + pad, w_row=cin + pad,
                                 w_group=cout * (cin + pad) if groups else 0, y_row=cout + pad)

    def forward(self, **kw):
        self.op.run(self.x, self.w, self.outs["y"][1], bias=self.bias, residual=self.residual, offsets=self.offsets, pre=self.outs["pre"][1], **kw)

    def backward(self, **kw):
        self.op.backward(self.dy, self.x, self.w, pre=self.pre_in if self.act != "none" else None, offsets=self.offsets, dx=self.outs["dx"][1],
                         dw=self.outs["dw"][1], dbias=self.dbias, **kw)

    def want(self):
        """name -> (value, tolerance), rows of no group left out."""
        r, n_in, n_out = HALF[self.dtype], self.x.shape[1], self.w.shape[-2]
        x, dy, z_in = self.x.double(), self.dy.double(), self.pre_in.double()
        w = self.w.double() if self.offsets is not None else self.w.double()[None]
        bias = None if self.bias is None else self.bias.double().view(len(w), -1)
        f64 = dict(dtype=torch.float64, device="cuda")
        z, zt = torch.zeros(self.rows, n_out, **f64), torch.zeros(self.rows, n_out, **f64)
        dx, dxt = torch.zeros(self.rows, n_in, **f64), torch.zeros(self.rows, n_in, **f64)
        dw, dwt = torch.zeros_like(w), torch.zeros_like(w)
        db, dbt = torch.zeros(len(w), n_out, **f64), torch.zeros(len(w), n_out, **f64)
        dz, dzt, rz = dy, 0 * dy, 0.0
        if self.act != "none":
            s = act_ref(z_in, self.act)[1]
            dz = dy * s
            dzt, rz = dy.abs() * ((1 + z_in.abs()) * act_eval(z_in, self.act) + 2 * U), r
        for g, (a, b) in enumerate(self.spans):
            m = b - a
            if not m:
                continue
            z[a:b] = x[a:b] @ w[g].t()
            zt[a:b] = (n_in + 2) * U * (x[a:b].abs() @ w[g].abs().t())
            if bias is not None:
                z[a:b] += bias[g]
                zt[a:b] += U * (bias[g].abs() + z[a:b].abs())
            d, dt = dz[a:b], dzt[a:b] + rz * dz[a:b].abs()      # dz as the products see it
            dx[a:b], dxt[a:b] = d @ w[g], dt @ w[g].abs() + (n_out + 2) * U * (d.abs() @ w[g].abs())
            dw[g], dwt[g] = d.t() @ x[a:b], dt.t() @ x[a:b].abs() + (m + 2) * U * (d.abs().t() @ x[a:b].abs())
            db[g], dbt[g] = d.sum(0), dzt[a:b].sum(0) + (m + 2) * U * d.abs().sum(0)
        y = act_ref(z, self.act)[0]
        yt = 1.13 * zt + z.abs() * act_eval(z, self.act)
        if self.residual is not None:
            y = y + self.residual.double()
            yt = yt + 2 * U * y.abs()
        out = {"y": (y, yt), "pre": (z, zt), "dx": (dx, dxt), "dw": (dw.view(self.w.shape), dwt.view(self.w.shape)), "dbias": (db.view(self.dbias.shape), dbt.view(self.dbias.shape))}
        return {k: (v, t + (U if k == "dbias" else r) * (v.abs() + t) + 1e-37) for k, (v, t) in out.items()}

    def check(self, names):
        torch.cuda.synchronize()
        want = self.want()
        for name in names:
            buf, got = (self.dbias, self.dbias) if name == "dbias" else self.outs[name]
            v, tol = want[name]
            if name in ("y", "pre", "dx"):
                assert (got[~self.inside] == -7.0).all(), f"{name}: rows of no group were written"
                got, v, tol = got[self.inside], v[self.inside], tol[self.inside]
            assert torch.isfinite(got).all(), f"{name}: not finite"
            err = (got.double() - v).abs()
            worst = (err / tol).max().item() if err.numel() else 0.0
            assert worst <= 1, f"{name}: {worst:.2f} of the tolerance, {self.op.info}"
            if name != "dbias":
                assert untouched(*self.outs[name], -7.0), f"{name}: written outside its window"


SHAPES = [(1, 1, 1), (1, 8, 8), (2, 64, 128), (3, 5, 7), (16, 96, 64), (33, 128, 31), (64, 33, 128), (127, 129, 65), (128, 128, 128), (129, 200, 136),
          (257, 64, 264), (300, 777, 257), (70, 2048, 48), (1000, 72, 520)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,cout", SHAPES)
def test_linear(rows, cin, cout, dtype):
    c = Linear(rows, cin, cout, dtype, act=ACTS[(rows + cin) % 5], seed=rows)
    c.forward()
    c.check(["y", "pre"])
    c.backward()
    c.check(["dx", "dw", "dbias"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype):
    """Every activation, its derivative, with and without bias and residual; z up to about 30 in size."""
    for bias, residual in ((True, True), (False, False), (True, False)):
        c = Linear(96, 64, 136, dtype, act=act, bias=bias, residual=residual, scale=8.0, seed=3)
        c.pre_in.mul_(8)
        c.forward()
        c.backward()
        c.check(["y", "pre", "dx", "dw", "dbias"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (3, 0), (1, 1), (0, 1), (16, 4)])
def test_linear_windows(pad, shift, dtype):
    """Operands that are windows of larger tensors, at any element: nothing around them is read into a result or written."""
    for rows, cin, cout in ((70, 72, 136), (130, 40, 24), (5, 256, 128)):
        c = Linear(rows, cin, cout, dtype, act="gelu", pad=pad, shift=shift, seed=pad)
        c.forward()
        c.backward()
        c.check(["y", "pre", "dx", "dw", "dbias"])


OFFSETS = {
    "one": [0, 90], "even": [0, 30, 60, 90], "empty_first": [0, 0, 50, 90], "empty_last": [0, 50, 90, 90], "empty_all": [0, 0, 0, 0, 0],
    "single_rows": list(range(0, 91, 1)), "one_big": [0, 1, 2, 89, 90], "rows_outside": [7, 20, 20, 33, 80], "far_out": [-5, 20, 1000, 2000],
    "decreasing": [0, 40, 10, 60, 55, 90], "many": [0] * 70 + [13, 13, 40] + [41] * 80 + [90],
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(OFFSETS))
def test_experts(name, dtype):
    for cin, cout in ((64, 136), (37, 20)):
        c = Linear(90, cin, cout, dtype, act="silu", offsets=OFFSETS[name], seed=len(name))
        c.forward()
        c.check(["y", "pre"])
        c.backward()
        c.check(["dx", "dw", "dbias"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_experts_longer(dtype):
    """Groups of several tiles, uneven, in windows of larger tensors."""
    for pad in (0, 8):
        c = Linear(1500, 136, 264, dtype, act="gelu_tanh", offsets=[0, 700, 701, 701, 960, 1100, 1490], pad=pad, seed=9)
        c.forward()
        c.backward()
        c.check(["y", "pre", "dx", "dw", "dbias"])


def test_only_what_is_asked_for():
    c = Linear(200, 64, 72, "bf16", act="relu")
    want = c.want()
    for names in (["dx"], ["dw"], ["dbias"], ["dx", "dbias"]):
        got = {n: torch.full(want[n][0].shape, -7.0, dtype=torch.float32 if n == "dbias" else torch.bfloat16, device="cuda") for n in names}
        c.op.backward(c.dy, c.x if "dw" in names else None, c.w if "dx" in names else None, pre=c.pre_in, **got)
        torch.cuda.synchronize()
        for n in names:
            assert ((got[n].double() - want[n][0]).abs() <= want[n][1]).all(), (names, n)


def test_residual_in_place():
    c = Linear(100, 64, 72, "bf16", act="none")
    y = c.residual.clone()
    c.op.run(c.x, c.w, y, bias=c.bias, residual=y)
    torch.cuda.synchronize()
    v, tol = c.want()["y"]
    assert ((y.double() - v).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_gives_zero_gradients(dtype):
    dt = TYPES[dtype]
    for groups in (0, 3):
        lead = (groups,) if groups else ()
        op = B.StripeLinear(0, 40, 24, dtype, activation="silu", groups=groups)
        dw, db = torch.full(lead + (24, 40), -7.0, dtype=dt, device="cuda"), torch.full(lead + (24,), -7.0, device="cuda")
        none = torch.empty(0, 24, dtype=dt, device="cuda")
        offsets = torch.zeros(4, dtype=torch.int32, device="cuda") if groups else None
        op.backward(none, torch.empty(0, 40, dtype=dt, device="cuda"), torch.empty(lead + (24, 40), dtype=dt, device="cuda"), pre=none, offsets=offsets,
                    dw=dw, dbias=db)
        torch.cuda.synchronize()
        assert (dw == 0).all() and (db == 0).all()


def test_non_finite_values_stay_where_they_belong():
    """A row with an infinity and one with a NaN: their own results show it, every other one is what it is without them."""
    c = Linear(90, 64, 136, "bf16", act="relu", residual=False)
    c.forward()
    torch.cuda.synchronize()
    before = c.outs["y"][1].clone()
    c.x[3, 5], c.x[77, 0] = float("inf"), NAN
    c.forward()
    torch.cuda.synchronize()
    y = c.outs["y"][1]
    keep = torch.ones(90, dtype=torch.bool, device="cuda")
    keep[3] = keep[77] = False
    assert torch.equal(y[keep], before[keep])
    assert torch.isnan(y[77]).all()
    up = c.w[:, 5] > 0
    assert torch.isinf(y[3][up]).all() and (y[3][~up & (c.w[:, 5] < 0)] == 0).all()


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
def test_gradients_against_differences(act):
    """The derivative of sum(y dy) along a direction, by central differences of the formulas in 64 bits.

    With steps h = 1e-5 the differences are off by h^2/6 of the third derivative (below 1e-9 of the terms) and by 64-bit roundings over h
    (1e-10 of them); the kernels' fp32 gradients by (n + 2) u of the terms, n <= 136: 2^-16 of the sum of |terms| covers all."""
    c = Linear(48, 64, 136, "f32", act=act, offsets=[0, 20, 20, 48], residual=False)
    c.forward()
    c.op.backward(c.dy, c.x, c.w, pre=c.outs["pre"][1], offsets=c.offsets, dx=c.outs["dx"][1], dw=c.outs["dw"][1], dbias=c.dbias)
    torch.cuda.synchronize()
    g = torch.Generator(device="cuda").manual_seed(1)

    def value(x, w, b):
        return sum((act_ref(x[s:e] @ w[i].t() + b[i], act)[0] * c.dy[s:e].double()).sum() for i, (s, e) in enumerate(c.spans))

    at = [c.x.double(), c.w.double(), c.bias.double()]
    for k, grad in enumerate((c.outs["dx"][1], c.outs["dw"][1], c.dbias)):
        v = torch.randn(at[k].shape, generator=g, device="cuda", dtype=torch.float64)
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + 1e-5 * v, at[k] - 1e-5 * v
        slope = (value(*up) - value(*down)) / 2e-5
        got, terms = (grad.double() * v).sum(), (grad.double() * v).abs().sum()
        assert abs(got - slope) <= 2.0 ** -16 * terms


def _replays(run, outs, change):
    """Captures run() into a graph and compares replays, with eager work between them, with eager results."""
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        run()
    for _ in range(3):
        change()
        run()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        for o, v in zip(outs, want):
            assert torch.equal(o, v)


def test_captured_and_replayed():
    c = Linear(300, 128, 136, "bf16", act="silu", offsets=[0, 100, 100, 300])
    c.op.set_workspace(torch.empty(c.op.workspace_bytes, dtype=torch.uint8, device="cuda"))
    outs = [c.outs[n][1] for n in ("y", "pre", "dx", "dw")] + [c.dbias]
    _replays(lambda: (c.forward(), c.backward()), outs, lambda: (c.x.mul_(0.5), c.offsets.copy_(torch.tensor([0, 50, 220, 300], dtype=torch.int32))))
    n = Norm(300, 1000, "bf16")
    outs = [n.y, n.mean, n.rstd, n.dx, n.dgamma, n.dbeta]
    _replays(lambda: (n.forward(), n.backward()), outs, lambda: n.x.mul_(0.5))


def test_capture_without_workspace_is_refused():
    c = Linear(300, 128, 136, "bf16", act="silu", residual=False)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    spare = torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph, stream=side):
        spare.add_(1)
        c.forward()                                    # needs none
        with pytest.raises(B.StripeError) as e:
            c.backward()
    assert e.value.status == 7
    graph.replay()
    torch.cuda.synchronize()
    c.check(["y", "pre"])
    c.backward()                                       # not captured: allocates
    c.check(["dx", "dw", "dbias"])


def test_runs_on_the_current_stream_and_on_a_given_one():
    c = Linear(128, 128, 128, "bf16", act="gelu")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.forward()
        c.backward()
    side.synchronize()
    c.check(["y", "pre", "dx", "dw", "dbias"])
    c.forward(stream=side.cuda_stream)
    c.check(["y", "pre"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart(dtype):
    """Row strides beyond the 32-bit offsets of a tile's loads."""
    c = Linear(40, 72, 136, dtype, act="gelu", pad=(1 << 20) + 8, seed=2)
    c.forward()
    c.backward()
    c.check(["y", "pre", "dx", "dw", "dbias"])


@pytest.mark.parametrize("few", [0, 1])
def test_f32_in_parts_with_infinities_nan_and_the_largest_values(few, monkeypatch):
    """What three bf16 parts cannot hold is computed again in fp32: every value and every neighbour as the formula has them."""
    monkeypatch.setenv("STRIPE_TUNE", f"product_few={few}")
    c = Linear(40, 72, 136, "f32", act="none", bias=False, residual=False, pad=(1 << 20) + 8, seed=4)
    assert ("rows" if few else "parts") in c.op.info["forward"] and "parts" in c.op.info["input_grad"] and "parts" in c.op.info["weight_grad"]
    big = torch.finfo(torch.float32).max
    c.x[3, 5], c.x[7, 0], c.x[11, 2], c.x[12, 3], c.x[13, 4] = float("inf"), NAN, big, -big, big
    c.x[13, 6], c.x[14] = float("-inf"), 0.0
    c.w[20, 2] = 1.0                                   # big times one is still finite
    c.dy[9, 8], c.dy[10, 8] = big, float("-inf")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    x, w, dy = c.x.double(), c.w.double(), c.dy.double()

    def same(got, a, b):
        v, terms = a @ b, a.abs() @ b.abs()
        tol = (a.shape[1] + 2) * U * terms
        tol = tol + U * (v.abs() + tol) + 1e-37
        # Where the finite terms' sizes add up to the largest fp32 value (big times 1.5, say), fp32 sums of them overflow in some or every order and meet
        # what infinities there are: 64 bits say nothing about such a result.
        beyond = a.nan_to_num(0, 0, 0).abs() @ b.nan_to_num(0, 0, 0).abs() * (1 + (a.shape[1] + 2) * U) >= big
        finite, special = torch.isfinite(v) & ~beyond, ~torch.isfinite(v) & ~beyond
        assert (((got.double() - v).abs() <= tol) | ~finite).all()
        assert torch.equal(torch.isnan(got)[special], torch.isnan(v)[special])
        known = special & ~torch.isnan(v)
        assert (got[known].double() == v[known]).all()
        assert (finite | special).double().mean() > 0.9

    same(c.outs["y"][1], x, w.t())
    same(c.outs["dx"][1], dy, w)
    same(c.outs["dw"][1], dy.t(), x)


def test_many_groups_of_many_tiles():
    sizes = [(37 * i) % 211 for i in range(75)]
    offsets = np.concatenate([[3], 3 + np.cumsum(sizes)]).tolist()
    for dtype in ("bf16", "f32"):
        c = Linear(offsets[-1] + 20, 72, 200, dtype, act="silu", offsets=offsets, seed=6)
        c.forward()
        c.backward()
        c.check(["y", "pre", "dx", "dw", "dbias"])


def test_more_than_two_billion_elements():
    """y, dz and dx beyond 2^31 elements: the last rows and columns."""
    rows, cin, cout = 66000, 64, 32776
    g = torch.Generator(device="cuda").manual_seed(0)
    x, w = (torch.randn(n, cin, generator=g, device="cuda").to(torch.bfloat16) for n in (rows, cout))
    y, dy = (torch.empty(rows, cout, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dy.normal_(generator=g)
    pre, dx, dw = dy, torch.empty_like(x), torch.empty_like(w)
    op = B.StripeLinear(rows, cin, cout, "bf16", activation="relu")
    op.run(x, w, y)
    op.backward(dy, x, w, pre=pre, dx=dx, dw=dw)
    torch.cuda.synchronize()
    for part in (slice(0, 70), slice(rows - 70, rows)):
        z, terms = x[part].double() @ w.double().t(), x[part].double().abs() @ w.double().abs().t()
        tol = (cin + 2) * U * terms
        assert ((y[part].double() - z.clamp(min=0)).abs() <= tol + 2.0 ** -8 * (z.abs() + tol)).all()
        dz = dy[part].double().clamp(min=0)
        tol = (cout + 2) * U * (dz @ w.double().abs())
        assert ((dx[part].double() - dz @ w.double()).abs() <= tol + 2.0 ** -8 * ((dz @ w.double()).abs() + tol)).all()
    dz = dy[:, -9:].double().clamp(min=0)
    v, tol = dz.t() @ x.double(), (rows + 2) * U * (dz.t() @ x.double().abs())
    assert ((dw[-9:].double() - v).abs() <= tol + 2.0 ** -8 * (v.abs() + tol)).all()


@pytest.mark.parametrize("rows", [3, 64])
def test_weights_of_more_than_two_billion_elements(rows):
    cin, cout = 65544, 32776
    g = torch.Generator(device="cuda").manual_seed(0)
    w = torch.empty(cout, cin, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    x, dy = (torch.randn(rows, n, generator=g, device="cuda").to(torch.bfloat16) for n in (cin, cout))
    y, dx = torch.empty_like(dy), torch.empty_like(x)
    op = B.StripeLinear(rows, cin, cout, "bf16")
    op.run(x, w, y)
    op.backward(dy, x, w, dx=dx)
    torch.cuda.synchronize()
    for got, a, b in ((y[:, -40:], x, w[-40:].double().t()), (dx[:, -40:], dy, w[:, -40:].double())):
        v, tol = a.double() @ b, (a.shape[1] + 2) * U * (a.double().abs() @ b.abs())
        assert ((got.double() - v).abs() <= tol + 2.0 ** -8 * (v.abs() + tol)).all()


def test_two_layers_on_two_streams():
    a, b = Linear(700, 264, 520, "bf16", act="silu", seed=1), Linear(700, 264, 520, "bf16", act="silu", seed=2)
    a.backward()                                       # each has its own workspace from here on
    b.backward()
    torch.cuda.synchronize()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.forward(stream=s.cuda_stream)
        b.forward(stream=t.cuda_stream)
        a.backward(stream=s.cuda_stream)
        b.backward(stream=t.cuda_stream)
    for c in (a, b):
        c.check(["y", "pre", "dx", "dw", "dbias"])


def test_two_graphs_with_workspaces_of_their_own():
    cs = [Linear(300, 128, 136, "f32", act="gelu", seed=i) for i in range(2)]
    graphs = []
    for c in cs:
        c.op.set_workspace(torch.empty(c.op.workspace_bytes, dtype=torch.uint8, device="cuda"))
        c.backward()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            c.forward()
            c.backward()
        graphs.append(graph)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        for c in cs:
            c.x.mul_(0.5)
            for _, o in c.outs.values():
                o.fill_(-7.0)
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, (s, t)):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for c in cs:
            c.check(["y", "pre", "dx", "dw", "dbias"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations_of_large_values(act, dtype):
    """|z| >= 40: act(z) is z or 0 up to |z| e^-40 < 2^-50, act'(z) 1 or 0 up to (1 + |z|^3) e^-40 < 2^-40 or what a square past overflow must not
    turn into NaN; two roundings of fp32, one of the result's type."""
    z = torch.tensor([40.0, -40.0, 1e4, -1e4, 1e10, -1e10, 2e19, -2e19, 3e38, -3e38], device="cuda", dtype=TYPES[dtype])
    n = z.numel()
    op = B.StripeLinear(1, 1, n, dtype, activation=act)
    x, y = torch.ones(1, 1, dtype=z.dtype, device="cuda"), torch.zeros(1, n, dtype=z.dtype, device="cuda")
    dy, db = torch.ones_like(z)[None], torch.zeros(n, device="cuda")
    op.run(x, z[:, None], y)
    op.backward(dy, x, z[:, None], pre=z[None], dbias=db)
    torch.cuda.synchronize()
    one = torch.ones_like(z) if act == "none" else (z > 0).to(z.dtype)
    want = (z * one).double()
    assert ((y[0].double() - want).abs() <= 2.0 ** -50 + (2 * U + HALF[dtype]) * want.abs()).all(), y
    assert ((db.double() - one.double()).abs() <= 2.0 ** -40 + 2 * U).all(), db


def test_wrapper_refuses_host_tensors():
    c = Linear(16, 32, 48, "bf16")
    with pytest.raises(ValueError, match="x: expected"):
        c.op.run(c.x.cpu(), c.w, c.outs["y"][1])


# ---- layer norm ------------------------------------------------------------------
class Norm:
    """n: additions one after the other in a sum over a row -- at most 32 in a lane (features / 1024 where rows are longer than that), then
    a tree over 64 lanes and a sum over at most 16 wavefronts."""

    def __init__(self, rows, features, dtype, eps=1e-5, affine=True, pad=0, shift=0, mean=0.25, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt, self.dtype, self.eps, self.affine = TYPES[dtype], dtype, eps, affine

        def make(v):
            view = window((rows, features), features + pad, dt, shift)[1]
            view.copy_(v.to(dt))
            return view

        self.x = make(torch.randn(rows, features, generator=g, device="cuda") * 1.5 + mean)
        self.dy = make(torch.randn(rows, features, generator=g, device="cuda"))
        self.gamma, self.beta = (torch.randn(features, generator=g, device="cuda") for _ in range(2)) if affine else (None, None)
        self.bufs = {n: window((rows, features), features + pad, dt, shift, -7.0) for n in ("y", "dx")}
        self.y, self.dx = self.bufs["y"][1], self.bufs["dx"][1]
        self.mean, self.rstd = (torch.full((rows,), -7.0, device="cuda") for _ in range(2))
        self.dgamma, self.dbeta = (torch.full((features,), -7.0, device="cuda") for _ in range(2))
        self.op = B.StripeNorm(rows, features, dtype, eps=eps, x_row=features + pad, y_row=features + pad)
        self.n = 32 + 6 + 16 + features // 1024 + 2

    def forward(self):
        self.op.run(self.x, self.y, gamma=self.gamma, beta=self.beta, mean=self.mean, rstd=self.rstd)

    def backward(self):
        self.op.backward(self.dy, self.x, self.mean, self.rstd, gamma=self.gamma, dx=self.dx, dgamma=self.dgamma, dbeta=self.dbeta)

    def check_forward(self):
        torch.cuda.synchronize()
        x, n, r = self.x.double(), self.n, HALF[self.dtype]
        m = x.mean(1, keepdim=True)
        d = x - m
        var = (d * d).mean(1, keepdim=True) + self.eps
        s = var ** -0.5
        em = n * U * x.abs().mean(1, keepdim=True) + U * m.abs()
        es = s * ((n + 4) * U + em * em / var + 2 * U * em * d.abs().mean(1, keepdim=True) / var + 4 * U)
        h = d * s
        eh = (em + U * d.abs()) * s + d.abs() * es + 2 * U * h.abs()
        gamma, beta = (self.gamma.double(), self.beta.double()) if self.affine else (1.0, 0.0)
        y = h * gamma + beta
        ey = eh * abs(gamma) + U * ((h * gamma).abs() + y.abs())
        for name, got, v, tol in (("mean", self.mean, m[:, 0], em[:, 0] + U * m[:, 0].abs()), ("rstd", self.rstd, s[:, 0], es[:, 0] + U * s[:, 0]),
                                  ("y", self.y, y, ey + r * (y.abs() + ey) + 1e-37)):
            assert torch.isfinite(got).all() and ((got.double() - v).abs() <= tol).all(), f"{name}: {((got.double() - v).abs() / tol).max()}"
        assert untouched(*self.bufs["y"], -7.0)

    def check_backward(self):
        """With the stored mean and rstd as inputs."""
        torch.cuda.synchronize()
        x, dy, n, r, rows = self.x.double(), self.dy.double(), self.n, HALF[self.dtype], self.x.shape[0]
        m, s = self.mean.double()[:, None], self.rstd.double()[:, None]
        h, g = (x - m) * s, dy * (self.gamma.double() if self.affine else 1.0)
        mg, mgh = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
        emg, emgh = (n + 2) * U * g.abs().mean(1, keepdim=True), (n + 6) * U * (g * h).abs().mean(1, keepdim=True)
        dx = s * (g - mg - h * mgh)
        edx = s * (8 * U * (g.abs() + mg.abs() + (h * mgh).abs()) + emg + h.abs() * emgh)
        dg, db = (dy * h).sum(0), dy.sum(0)
        for name, got, v, tol in (("dx", self.dx, dx, edx + r * (dx.abs() + edx) + 1e-37), ("dgamma", self.dgamma, dg, (rows + 6) * U * (dy * h).abs().sum(0)),
                                  ("dbeta", self.dbeta, db, (rows + 2) * U * dy.abs().sum(0))):
            assert torch.isfinite(got).all() and ((got.double() - v).abs() <= tol + 1e-37).all(), f"{name}: {((got.double() - v).abs() / tol).max()}"
        assert untouched(*self.bufs["dx"], -7.0)


NORM_SHAPES = [(1, 1), (1, 8), (1, 4096), (2, 3), (3, 64), (5, 119), (7, 511), (4, 512), (9, 513), (64, 1000), (33, 2048), (17, 2049), (1000, 72), (12, 4100),
               (6, 8192), (3, 8193), (2, 16384), (3, 16391), (2, 32768), (2, 33000), (3, 70001), (4099, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,features", NORM_SHAPES)
def test_norm(rows, features, dtype):
    c = Norm(rows, features, dtype, affine=(rows + features) % 3 != 0, seed=features, eps=1e-5 if features > 1 else 0.5)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (5, 3)])
def test_norm_windows(pad, shift, dtype):
    for rows, features in ((20, 520), (6, 3001), (2, 40000)):
        c = Norm(rows, features, dtype, pad=pad, shift=shift)
        c.forward()
        c.check_forward()
        c.backward()
        c.check_backward()


def test_norm_of_rows_far_from_zero():
    """A mean a thousand times the spread: the squared distances are from the mean, not from zero."""
    c = Norm(40, 3000, "f32", mean=1000.0)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


def test_norm_in_place_and_parts():
    c = Norm(30, 1000, "bf16")
    c.forward()
    want = c.y.clone()
    x = c.x.clone()
    c.op.run(x, x, gamma=c.gamma, beta=c.beta)
    c.backward()
    whole = [c.dx.clone(), c.dgamma.clone(), c.dbeta.clone()]
    torch.cuda.synchronize()
    assert torch.equal(x, want)
    for keep in range(3):
        got = [torch.empty_like(t) if i == keep else None for i, t in enumerate(whole)]
        c.op.backward(c.dy, c.x, c.mean, c.rstd, gamma=c.gamma, dx=got[0], dgamma=got[1], dbeta=got[2])
        torch.cuda.synchronize()
        assert torch.equal(got[keep], whole[keep])


@pytest.mark.parametrize("features", [40, 40000])
def test_norm_without_rows(features):
    op = B.StripeNorm(0, features, "f32")
    dg, db = (torch.full((features,), -7.0, device="cuda") for _ in range(2))
    none, row = torch.empty(0, features, device="cuda"), torch.empty(0, device="cuda")
    op.backward(none, none, row, row, dx=none, dgamma=dg, dbeta=db)
    torch.cuda.synchronize()
    assert (dg == 0).all() and (db == 0).all()


def test_norm_gradient_against_differences():
    """As for the linear layer: 2^-16 of the terms; the sums here have at most 600 terms, whose (n + 6) u of sum |terms| is below that."""
    c = Norm(7, 600, "f32")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    g = torch.Generator(device="cuda").manual_seed(1)

    def value(x, gamma, beta):
        d = x - x.mean(1, keepdim=True)
        return ((d * ((d * d).mean(1, keepdim=True) + c.eps) ** -0.5 * gamma + beta) * c.dy.double()).sum()

    at = [c.x.double(), c.gamma.double(), c.beta.double()]
    for k, grad in enumerate((c.dx, c.dgamma, c.dbeta)):
        v = torch.randn(at[k].shape, generator=g, device="cuda", dtype=torch.float64)
        up, down = list(at), list(at)
        up[k], down[k] = at[k] + 1e-5 * v, at[k] - 1e-5 * v
        slope, terms = (value(*up) - value(*down)) / 2e-5, (grad.double() * v).abs().sum()
        assert abs((grad.double() * v).sum() - slope) <= 2.0 ** -16 * terms


# ---- together ---------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_feed_forward_block(dtype):
    """A block as a model has it: out = x + W2 act(W1 norm(x) + b1) + b2, and every gradient, against the formulas in 64 bits that take the
    stored intermediate tensors (each operator alone is held to its own tolerance above).

    Relative 2-norms: a stored bf16 tensor is off by at most 2^-8 per element and passes two products and an activation; six such roundings
    lie between the input and the furthest gradient: 6 x 1.13 x 2^-8 = 0.027.  fp32: the roundings of sums of up to 700 terms, 700 u each: 6 x 700 u."""
    rows, c, f = 700, 264, 520
    dt, tol = TYPES[dtype], {"bf16": 6 * 1.13 * 2.0 ** -8, "f32": 6 * 700 * U}[dtype]
    g = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s, scale=1.0, dtype=dt: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)      # noqa: E731
    out = lambda *s, dtype=dt: torch.empty(*s, dtype=dtype, device="cuda")                                     # noqa: E731
    x, dout = new(rows, c), new(rows, c)
    w1, w2, b1, b2 = new(f, c, scale=c ** -0.5), new(c, f, scale=f ** -0.5), new(f, scale=0.1, dtype=torch.float32), new(c, scale=0.1, dtype=torch.float32)
    gamma, beta = 1 + new(c, scale=0.1, dtype=torch.float32), new(c, scale=0.1, dtype=torch.float32)
    norm, up, down = B.StripeNorm(rows, c, dtype), B.StripeLinear(rows, c, f, dtype, activation="gelu"), B.StripeLinear(rows, f, c, dtype)
    h, mean, rstd, z, a, y = out(rows, c), out(rows, dtype=torch.float32), out(rows, dtype=torch.float32), out(rows, f), out(rows, f), out(rows, c)
    norm.run(x, h, gamma=gamma, beta=beta, mean=mean, rstd=rstd)
    up.run(h, w1, a, bias=b1, pre=z)
    down.run(a, w2, y, bias=b2, residual=x)
    da, dh, dx = out(rows, f), out(rows, c), out(rows, c)
    dw1, dw2, db1, db2, dgamma, dbeta = out(f, c), out(c, f), *(out(n, dtype=torch.float32) for n in (f, c, c, c))
    down.backward(dout, a, w2, dx=da, dw=dw2, dbias=db2)
    up.backward(da, h, w1, pre=z, dx=dh, dw=dw1, dbias=db1)
    norm.backward(dh, x, mean, rstd, gamma=gamma, dx=dx, dgamma=dgamma, dbeta=dbeta)
    torch.cuda.synchronize()
    leaves = [t.double().requires_grad_() for t in (x, w1, w2, b1, b2, gamma, beta)]
    X, W1, W2, B1, B2, G, Bt = leaves
    d = X - X.mean(1, keepdim=True)
    hid = d * ((d * d).mean(1, keepdim=True) + 1e-5) ** -0.5 * G + Bt
    zz = hid @ W1.t() + B1
    Y = X + (zz * torch.special.ndtr(zz)) @ W2.t() + B2
    Y.backward(dout.double())
    ours = {"y": (y, Y.detach()), "dx": (dx.double() + dout.double(), X.grad), "dw1": (dw1, W1.grad), "dw2": (dw2, W2.grad), "db1": (db1, B1.grad),
            "db2": (db2, B2.grad), "dgamma": (dgamma, G.grad), "dbeta": (dbeta, Bt.grad)}
    for name, (got, v) in ours.items():
        rel = (got.double() - v).norm() / v.norm()
        assert rel <= tol, f"{name}: {rel:.2e}"


def test_norm_of_more_than_two_billion_elements():
    rows, features = (1 << 18) + 5, 8200
    x = torch.empty(rows, features, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(0))
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dbeta = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(features, device="cuda")
    op = B.StripeNorm(rows, features, "bf16")
    op.run(x, y, mean=mean, rstd=rstd)
    op.backward(y, x, mean, rstd, dx=dx, dgamma=torch.empty(features, device="cuda"), dbeta=dbeta)
    torch.cuda.synchronize()
    n = 32 + 6 + 16 + 8 + 2
    for part in (slice(0, 50), slice(rows - 50, rows)):
        xd = x[part].double()
        d = xd - xd.mean(1, keepdim=True)
        s = ((d * d).mean(1, keepdim=True) + 1e-5) ** -0.5
        # (n + 8) u relative to |d| + mean|x| bounds the statistics' share; one rounding
        tol = (n + 8) * U * s * (d.abs() + xd.abs().mean(1, keepdim=True)) * 2
        assert ((y[part].double() - d * s).abs() <= tol + 2.0 ** -8 * ((d * s).abs() + tol)).all()
        # dx of dy = y = h (rounded): s (y - mean y - h mean(y h))
        yd, h = y[part].double(), (xd - mean[part].double()[:, None]) * rstd[part].double()[:, None]
        want = rstd[part].double()[:, None] * (yd - yd.mean(1, keepdim=True) - h * (yd * h).mean(1, keepdim=True))
        tol = rstd[part].double()[:, None] * (n + 14) * U * (yd.abs() + yd.abs().mean(1, keepdim=True) + h.abs() * (2 + (yd * h).abs().mean(1, keepdim=True)))
        assert ((dx[part].double() - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all()
    v = y[:, -9:].double()
    assert ((dbeta[-9:].double() - v.sum(0)).abs() <= (rows + 2) * U * v.abs().sum(0)).all()
