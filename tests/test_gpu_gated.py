"""The gated unit on the GPU, forward and gradients, against its formulas in 64 bits.

Tolerances, u = 2^-24, r = the result type's half step (bf16 2^-8, fp32 2^-24), derived per element (act_eval: the relative error of evaluating an
activation, see test_gpu_layers):
  g, u     n terms added in any order: e = (n + 2) u sum |terms|
  y        act(g) u: 1.13 e_g |u| + |act(g)| e_u + 1.13 e_g e_u, evaluating act |g u| act_eval, two roundings of the product, one of the result
  dz       dg: |dy u| (1 + |g|) act_eval + 3 u |dg|;  du: |dy g| act_eval + 2 u |du|;  then rounded to the operands' type: r |dz|
  dx, dW   the terms' errors, (terms + 2) u sum |terms|, one rounding
"""
import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import ACTS, HALF, NAN, TYPES, U, act_eval, act_ref, bounds, untouched, window

pytestmark = pytest.mark.gpu


class Gated:
    def __init__(self, rows, cin, cout, dtype, act="silu", offsets=None, pad=0, shift=0, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt, self.dtype, self.act, self.rows, self.n = TYPES[dtype], dtype, act, rows, cout
        groups = len(offsets) - 1 if offsets is not None else 0
        lead = (groups,) if groups else ()

        def make(*shape, s=1.0):
            _, v = window(shape, shape[-1] + pad, dt, shift)
            v.copy_((torch.randn(*shape, generator=g, device="cuda") * s).to(dt))
            return v

        self.x, self.w = make(rows, cin), make(*lead, 2 * cout, cin, s=cin ** -0.5)
        self.dy, self.pre_in = make(rows, cout), make(rows, 2 * cout, s=1.5)
        self.offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda") if groups else None
        self.spans = bounds(offsets, rows) if groups else [(0, rows)]
        self.inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
        for a, b in self.spans:
            self.inside[a:b] = True
        for t in (self.x, self.dy, self.pre_in):
            t[~self.inside] = NAN                      # rows of no group are nobody's
        self.outs = {name: window(shape, shape[-1] + pad, dt, shift, -7.0)
                     for name, shape in (("y", (rows, cout)), ("pre", (rows, 2 * cout)), ("dx", (rows, cin)), ("dw", lead + (2 * cout, cin)))}
        self.op = B.StripeGated(rows, cin, cout, dtype, activation=act, groups=groups, x_row=cin + pad, w_row=cin + pad,
                                w_group=2 * cout * (cin + pad) if groups else 0, y_row=cout + pad, pre_row=2 * cout + pad)

    def forward(self, pre=True, **kw):
        self.op.run(self.x, self.w, self.outs["y"][1], offsets=self.offsets, pre=self.outs["pre"][1] if pre else None, **kw)

    def backward(self, **kw):
        self.op.backward(self.dy, self.x, self.w, self.pre_in, offsets=self.offsets, dx=self.outs["dx"][1], dw=self.outs["dw"][1], **kw)

    def want(self):
        """name -> (value, tolerance), rows of no group left out."""
        r, cin, n = HALF[self.dtype], self.x.shape[1], self.n
        x, dy, pre = self.x.double(), self.dy.double(), self.pre_in.double()
        w = self.w.double() if self.offsets is not None else self.w.double()[None]
        z, zt = torch.zeros_like(pre), torch.zeros_like(pre)
        dx, dxt, dw, dwt = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w)
        g, u = pre[:, :n], pre[:, n:]
        value, slope = act_ref(g, self.act)
        ev = act_eval(g, self.act)
        dz = torch.cat([dy * u * slope, dy * value], 1)
        dzt = torch.cat([(dy * u).abs() * (1 + g.abs()) * ev, (dy * g).abs() * ev], 1) + 3 * U * dz.abs()
        dzt = dzt + r * (dz.abs() + dzt)
        for e, (a, b) in enumerate(self.spans):
            if a == b:
                continue
            z[a:b], zt[a:b] = x[a:b] @ w[e].t(), (cin + 2) * U * (x[a:b].abs() @ w[e].abs().t())
            dx[a:b] = dz[a:b] @ w[e]
            dxt[a:b] = (dzt[a:b] + (2 * n + 2) * U * dz[a:b].abs()) @ w[e].abs() + r * dx[a:b].abs()
            dw[e] = dz[a:b].t() @ x[a:b]
            dwt[e] = (dzt[a:b] + (b - a + 2) * U * dz[a:b].abs()).t() @ x[a:b].abs() + r * dw[e].abs()
        g, u, gt, ut = z[:, :n], z[:, n:], zt[:, :n], zt[:, n:]
        value = act_ref(g, self.act)[0]
        yt = 1.13 * gt * u.abs() + value.abs() * ut + 1.13 * gt * ut + (g * u).abs() * act_eval(g, self.act) + 2 * U * (value * u).abs()
        y = value * u
        lead = self.w.shape
        return {"y": (y, yt + r * (y.abs() + yt)), "pre": (z, zt + r * (z.abs() + zt)), "dx": (dx, dxt * (1 + r)), "dw": (dw.view(lead), dwt.view(lead) * (1 + r))}

    def check(self, names=("y", "pre", "dx", "dw")):
        want = self.want()
        for name in names:
            buf, got = self.outs[name]
            value, tol = want[name]
            if name != "dw":
                assert (got[~self.inside] == -7.0).all(), f"{name}: a row of no group was written"
                got, value, tol = got[self.inside], value[self.inside], tol[self.inside]
            off = (got.double() - value).abs()
            bad = ~(off <= tol + 1e-35)
            assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / (tol + 1e-35)).max()):.2f} of the tolerance"
            assert untouched(*self.outs[name], -7.0), f"{name}: written outside its rows"


SIZES = [(1, 8, 1), (1, 64, 8), (3, 40, 17), (16, 512, 96), (17, 520, 33), (65, 64, 64), (130, 200, 129), (300, 333, 257), (257, 1024, 130)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_values_and_gradients(size, dtype):
    t = Gated(*size, dtype)
    t.forward()
    t.backward()
    t.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activations(act, dtype):
    t = Gated(70, 96, 72, dtype, act=act, seed=1)
    t.forward()
    t.backward()
    t.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (3, 1), (1, 0), (0, 5)])
@pytest.mark.parametrize("rows", [5, 150])
def test_strides_and_alignments(rows, pad, shift, dtype):
    t = Gated(rows, 136, 100, dtype, pad=pad, shift=shift, seed=2)
    t.forward()
    t.backward()
    t.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offsets", [[0, 0], [0, 90], [0, 10, 10, 64, 90], [5, 40, 20, 200, 80], [90, 90, 90], [-3, 1, 2, 3, 4, 5, 6, 7, 60]], ids=str)
def test_groups(offsets, dtype):
    t = Gated(90, 72, 48, dtype, offsets=offsets, seed=3)
    t.forward()
    t.backward()
    t.check()


@pytest.mark.parametrize("tile", range(4))
@pytest.mark.parametrize("splits", [1, 3])
def test_every_tile(monkeypatch, tile, splits):
    monkeypatch.setenv("STRIPE_TUNE", f"product_tile={tile},product_splits={splits},product_few=0")
    for size in ((300, 640, 200), (70, 1000, 77)):
        t = Gated(*size, "bf16", seed=4)
        t.forward()
        t.backward()
        t.check()
    t = Gated(200, 512, 136, "bf16", offsets=[0, 30, 170, 171, 200], seed=5)
    t.forward()
    t.check(("y", "pre"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cin,offsets", [(1, 4096, None), (40, 1000, None), (30, 264, [0, 3, 3, 20, 30])])
def test_few_rows(monkeypatch, rows, cin, offsets, dtype):
    monkeypatch.setenv("STRIPE_TUNE", "product_few=1")
    t = Gated(rows, cin, 83, dtype, offsets=offsets, seed=6)
    assert "product_rows" in t.op.info["forward"]
    t.forward()
    t.check(("y", "pre"))


def test_fp32_in_parts(monkeypatch):
    monkeypatch.setenv("STRIPE_TUNE", "product_tile=1,product_few=0")
    t = Gated(150, 256, 100, "f32", seed=7)
    assert "parts" in t.op.info["forward"]
    t.forward()
    t.backward()
    t.check()


def test_without_pre_and_single_gradients():
    t = Gated(100, 128, 64, "bf16", seed=8)
    t.forward(pre=False)
    assert (t.outs["pre"][0] == -7.0).all()
    t.op.backward(t.dy, t.x, t.w, t.pre_in, dx=t.outs["dx"][1])
    t.check(("y", "dx"))
    assert (t.outs["dw"][0] == -7.0).all()
    t.op.backward(t.dy, t.x, None, t.pre_in, dw=t.outs["dw"][1])
    t.check(("dw",))


def test_no_rows():
    t = Gated(0, 64, 32, "bf16")
    t.forward()
    t.backward()
    assert (t.outs["dw"][1] == 0).all()


def test_infinities_and_nan_go_the_formulas_way():
    t = Gated(4, 64, 16, "bf16", act="silu", seed=9)
    t.x[0, 0], t.x[1, 0] = NAN, float("inf")
    t.forward()
    z = t.x.double() @ t.w.double().t()
    y = act_ref(z[:, :16], "silu")[0] * z[:, 16:]
    got = t.outs["y"][1].double()
    assert torch.isnan(got[0]).all() and torch.equal(torch.isnan(got[1]), torch.isnan(y[1])) and torch.isfinite(got[2:]).all()
    fine = ~torch.isnan(y[1])
    assert torch.equal(torch.isinf(got[1][fine]), torch.isinf(y[1][fine]))


def test_gradient_against_differences():
    """d/dt of sum(dy y(x + t d, W + t e)) at 0, by differences of the forward pass in fp32.  With step h the difference is off by h^2 / 6 times the third
    derivative -- of z^2-like growth in values of size 1: at most 10 sum |terms| -- and by the sums' errors over h."""
    rows, cin, n, h = 40, 48, 24, 2.0 ** -7
    t = Gated(rows, cin, n, "f32", act="gelu", seed=10)
    t.forward()
    t.pre_in.copy_(t.outs["pre"][1])
    t.backward()
    g = torch.Generator(device="cuda").manual_seed(11)
    d, e = (torch.randn(rows, cin, generator=g, device="cuda") * cin ** -0.5, torch.randn(2 * n, cin, generator=g, device="cuda") / cin)

    def total(s):
        y = torch.empty(rows, n, device="cuda")
        t.op.run((t.x + s * d).contiguous(), (t.w + s * e).contiguous(), y)
        return float((t.dy.double() * y.double()).sum())

    slope = float((t.outs["dx"][1].double() * d.double()).sum() + (t.outs["dw"][1].double() * e.double()).sum())
    scale = float((t.dy.abs() * (1 + t.outs["y"][1].abs())).sum())
    assert abs((total(h) - total(-h)) / (2 * h) - slope) <= 10 * scale * h * h / 6 + scale * (cin + 64) * U / h


def test_streams_graphs_and_repeats():
    """The same bits on a stream of its own, from a captured graph (replayed among eager work), and from two handles at once."""
    t = Gated(300, 256, 136, "bf16", seed=12)
    ws = torch.empty(t.op.workspace_bytes, dtype=torch.uint8, device="cuda")
    t.op.set_workspace(ws)
    t.forward()
    t.backward()
    want = {k: v[1].clone() for k, v in t.outs.items()}
    side = torch.cuda.Stream()
    other = Gated(300, 256, 136, "bf16", seed=12)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other.forward()
        other.backward()
    t.forward()
    t.backward()
    torch.cuda.synchronize()
    for k, v in want.items():
        assert torch.equal(v, t.outs[k][1]) and torch.equal(v, other.outs[k][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.forward()
        t.backward()
    for _ in range(3):
        for v in t.outs.values():
            v[0].fill_(-7.0)
        graph.replay()
        other.forward()
        torch.cuda.synchronize()
        for k, v in want.items():
            assert torch.equal(v, t.outs[k][1])


def test_a_first_call_under_capture_is_refused():
    t = Gated(300, 256, 136, "bf16", seed=13)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(B.StripeError):
            t.backward()
        t.x.add_(0)
    t.backward()
    t.check(("dx", "dw"))


def test_wrapper_refuses_other_tensors():
    t = Gated(20, 64, 32, "bf16", seed=14)
    y = t.outs["y"][1]
    for args in ((t.x.float(), t.w, y), (t.x[:, :32], t.w, y), (t.x, t.w[:32], y), (t.x, t.w, y[:10]), (t.x.cpu(), t.w, y)):
        with pytest.raises(ValueError):
            t.op.run(*args)
    with pytest.raises(ValueError):
        t.op.run(t.x, t.w, y, pre=torch.empty(20, 32, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(B.StripeError):
        t.op.run(t.x, t.w, y, offsets=torch.zeros(1, dtype=torch.int32, device="cuda"))
    with pytest.raises(B.StripeError):
        t.op.backward(t.dy, t.x, t.w, t.pre_in, dx=t.x)


@pytest.mark.parametrize("offsets", [None, [0, 0, 300, 300, 1000, 4000, 4001, 4400, 4350], list(range(0, 4352, 68))], ids=["dense", "9", "64"])
@pytest.mark.parametrize("cin", [8, 64, 328])
def test_more_tiles_than_compute_units(monkeypatch, cin, offsets):
    """Several tiles of 256 x 256 for each compute unit, dense and with groups."""
    monkeypatch.setenv("STRIPE_TUNE", "product_tile=0,product_splits=1,product_few=0")
    t = Gated(4360, cin, 2200 if offsets is None else 1100, "bf16", offsets=offsets, seed=15)
    assert "256x256" in t.op.info["forward"]
    t.forward()
    t.backward()
    t.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_buffers_beyond_32_bits(dtype):
    """Rows of every buffer so far apart that the last lies more than 2^32 elements in."""
    rows, cin, n, dt = 90, 40, 48, TYPES[dtype]
    far = (1 << 32) // 85
    t = Gated(rows, cin, n, dtype, seed=16)

    def spread(v, like):
        s = torch.empty(v.shape[0] * far, dtype=dt, device="cuda").as_strided(v.shape, (far, 1))
        return s.copy_(v) if like else s

    op = B.StripeGated(rows, cin, n, dtype, x_row=far, w_row=far, y_row=far, pre_row=far)
    x, w, dy, pre_in = (spread(v, True) for v in (t.x, t.w, t.dy, t.pre_in))
    y, pre, dx, dw = (spread(t.outs[k][1], False) for k in ("y", "pre", "dx", "dw"))
    op.run(x, w, y, pre=pre)
    op.backward(dy, x, w, pre_in, dx=dx, dw=dw)
    for k, v in (("y", y), ("pre", pre), ("dx", dx), ("dw", dw)):
        t.outs[k][1].copy_(v)
    t.check()


def test_experts_far_apart_and_many_of_their_tiles():
    """Weight gradients whose matrices' tiles are spread over the XCDs, matrices beyond 2^32 elements, groups without rows."""
    rows, cin, n, groups = 700, 520, 1100, 5
    offsets = [0, 0, 500, 512, 512, 700]
    far = 1 << 30
    t = Gated(rows, cin, n, "bf16", offsets=offsets, seed=17)
    w, dw = (torch.empty(groups * far, dtype=torch.bfloat16, device="cuda").as_strided((groups, 2 * n, cin), (far, cin, 1)) for _ in range(2))
    w.copy_(t.w)
    op = B.StripeGated(rows, cin, n, "bf16", groups=groups, w_group=far)
    op.run(t.x, w, t.outs["y"][1], offsets=t.offsets, pre=t.outs["pre"][1])
    op.backward(t.dy, t.x, w, t.pre_in, offsets=t.offsets, dx=t.outs["dx"][1], dw=dw)
    t.outs["dw"][1].copy_(dw)
    t.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups", [65, 130, 4096])
def test_more_groups_than_a_wavefront_has_lanes(groups, dtype):
    rows = 600
    ends = [0] + sorted(int(v) for v in torch.randint(0, rows + 1, (groups - 1,), generator=torch.Generator().manual_seed(groups))) + [rows]
    t = Gated(rows, 24, 20, dtype, offsets=ends, seed=18)
    t.forward()
    t.backward()
    t.check()


@pytest.mark.parametrize("offsets", [None, [0, 30, 30, 200, 333]], ids=["dense", "groups"])
@pytest.mark.parametrize("size", [(333, 777, 130), (333, 70, 67), (340, 1, 5)], ids=lambda s: "x".join(map(str, s)))
def test_rows_copied_to_whole_pieces(monkeypatch, size, offsets):
    """bf16 rows that are no multiple of 16 bytes, with strides of their own."""
    monkeypatch.setenv("STRIPE_TUNE", "layers_copy=1,product_few=0")
    t = Gated(*size, "bf16", offsets=offsets, pad=3, shift=1, seed=19)
    assert all(v.endswith("_copied") for k, v in t.op.info.items() if k != "workspace_bytes")
    t.forward()
    t.backward()
    t.check()


def test_rows_that_are_no_whole_pieces_at_sizes_of_either_kind():
    """Whichever way the estimates send them: these sizes through registers, larger ones by copies."""
    t = Gated(1500, 1023, 1000, "bf16", seed=20)
    t.forward()
    t.backward()
    t.check()
    t = Gated(4100, 1324, 2000, "bf16", seed=21)
    assert t.op.info["forward"].endswith("_copied")
    t.forward()
    t.backward()
    t.check()
    assert not B.StripeGated(64, 63, 64, "bf16").info["forward"].endswith("_copied")
