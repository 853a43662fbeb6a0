"""The cross entropy of a linear head on the GPU, forward and gradients, against its formulas in 64 bits.

Tolerances, u = 2^-24, r = the result type's half step, derived per element:
  z        n terms added in any order: e = (n + 2) u sum |terms|
  lse      the largest e of its row (lse is 1-Lipschitz in z); each exponential's argument is rounded and scaled: 3 |z - lse| + 8 roundings, weighted with p;
           sums of at most 32 + classes / 256 steps, each with an exponential and a product more: 8 u each; the logarithm and its addition: 3 u (1 + |lse|)
  loss     the same, e of the target's z, and one rounding
  dz       p (dloss + dlse): p (e + u |lse| + 3 u |z - lse| + 8 u), 3 u of the result; rounded to the operands' type: r |dz|
  dx, dW   the terms' errors, (terms + 2) u sum |terms| (dx: one more for each piece of the vocabulary), one rounding
"""
import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import HALF, NAN, TYPES, U, untouched, window

pytestmark = pytest.mark.gpu
IGNORED = (-1, -100, 1 << 30)


class Xent:
    def __init__(self, rows, cin, classes, dtype, ignored=0.2, pad=0, shift=0, seed=0, dloss=True, dlse=True, scale=2.0, pieces=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt, self.dtype, self.shape, self.pieces = TYPES[dtype], dtype, (rows, cin, classes), pieces

        def make(*shape, s=1.0):
            _, v = window(shape, shape[-1] + pad, dt, shift)
            v.copy_((torch.randn(*shape, generator=g, device="cuda") * s).to(dt))
            return v

        self.x, self.w = make(rows, cin, s=scale), make(classes, cin, s=cin ** -0.5)
        target = torch.randint(0, classes, (rows,), generator=g, device="cuda")
        out = torch.rand(rows, generator=g, device="cuda") < ignored
        bad = torch.tensor(IGNORED + (classes,), device="cuda")[torch.randint(0, 4, (rows,), generator=g, device="cuda")]
        self.targets = torch.where(out, bad, target).to(torch.int32)
        self.counts = ~out
        self.x[out] = NAN                          # rows that do not count are not read
        self.dloss = torch.randn(rows, generator=g, device="cuda") if dloss else None
        self.dlse = torch.randn(rows, generator=g, device="cuda") if dlse else None
        for t in (self.dloss, self.dlse):
            if t is not None:
                t[out] = NAN
        self.loss, self.lse = torch.full((rows,), -7.0, device="cuda"), torch.full((rows,), -7.0, device="cuda")
        self.outs = {"dx": window((rows, cin), cin + pad, dt, shift, -7.0), "dw": window((classes, cin), cin + pad, dt, shift, -7.0)}
        self.op = B.StripeXent(rows, cin, classes, dtype, x_row=cin + pad, w_row=cin + pad)
        z = self.x.double() @ self.w.double().t()
        self.z = z[self.counts]
        self.lse_ref = torch.logsumexp(self.z, 1)

    def forward(self, **kw):
        self.op.run(self.x, self.w, self.targets, self.loss, self.lse, **kw)

    def lse_in(self):
        lse = torch.full((self.shape[0],), NAN, device="cuda")
        lse[self.counts] = self.lse_ref.float()
        return lse

    def backward(self, **kw):
        self.op.backward(self.x, self.w, self.targets, self.lse_in(), dloss=self.dloss, dlse=self.dlse, dx=self.outs["dx"][1], dw=self.outs["dw"][1], **kw)

    def check_forward(self):
        rows, cin, classes = self.shape
        c, z, lse = self.counts, self.z, self.lse_ref
        assert (self.loss[~c] == 0).all() and (self.lse[~c] == 0).all()
        e = (cin + 2) * U * (self.x[c].double().abs() @ self.w.double().abs().t())
        d = z - lse[:, None]
        tol = e.max(1).values + (d.exp() * (3 * d.abs() + 8) * U).sum(1) + (32 + classes / 256) * 8 * U + 3 * U * (1 + lse.abs())
        off = (self.lse[c].double() - lse).abs()
        assert (off <= tol).all(), f"lse: {float((off / tol).max()):.2f} of the tolerance"
        t = self.targets[c].long()[:, None]
        tol = tol + e.gather(1, t)[:, 0] + U * (lse - z.gather(1, t)[:, 0]).abs()
        off = (self.loss[c].double() - (lse - z.gather(1, t)[:, 0])).abs()
        assert (off <= tol).all(), f"loss: {float((off / tol).max()):.2f} of the tolerance"

    def check_backward(self, names=("dx", "dw")):
        (rows, cin, classes), r, c = self.shape, HALF[self.dtype], self.counts
        x, w, z, lse = self.x[c].double(), self.w.double(), self.z, self.lse_ref[:, None]
        one = self.dloss[c].double() if self.dloss is not None else torch.ones(len(z), dtype=torch.float64, device="cuda")
        both = one + self.dlse[c].double() if self.dlse is not None else one
        e = (cin + 2) * U * (x.abs() @ w.abs().t())
        p = torch.exp(z - lse)
        dz = p * both[:, None]
        dz.scatter_add_(1, self.targets[c].long()[:, None], -one[:, None])
        size = p * both.abs()[:, None]
        size.scatter_add_(1, self.targets[c].long()[:, None], one.abs()[:, None])
        dzt = p * both.abs()[:, None] * (e + U * lse.abs() + 3 * U * (z - lse).abs() + 8 * U) + 4 * U * size
        dzt = dzt + r * (dz.abs() + dzt)
        dx = torch.zeros(rows, cin, dtype=torch.float64, device="cuda")
        dxt = dx.clone()
        dx[c] = dz @ w
        dxt[c] = (dzt + (classes + 2 + self.pieces) * U * dz.abs()) @ w.abs() + r * dx[c].abs()
        dw = dz.t() @ x
        dwt = (dzt + (len(z) + 2) * U * dz.abs()).t() @ x.abs() + r * dw.abs()
        for name, value, tol in (("dx", dx, dxt), ("dw", dw, dwt)):
            if name not in names:
                continue
            buf, got = self.outs[name]
            off = (got.double() - value).abs()
            tol = tol * (1 + r) + 1e-35
            bad = ~(off <= tol)
            assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol).max()):.2f} of the tolerance"
            assert untouched(buf, got, -7.0), f"{name}: written outside its rows"


SIZES = [(1, 8, 1), (1, 64, 5), (2, 33, 130), (16, 256, 300), (17, 100, 65), (64, 512, 1000), (130, 72, 257), (300, 200, 515), (600, 64, 2049)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_values_and_gradients(size, dtype):
    t = Xent(*size, dtype)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (3, 1), (0, 5)])
def test_strides_and_alignments(pad, shift, dtype):
    t = Xent(150, 136, 400, dtype, pad=pad, shift=shift, seed=1)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pieces", [2, 3, 8])
def test_pieces_of_the_vocabulary(monkeypatch, pieces, dtype):
    monkeypatch.setenv("STRIPE_TUNE", f"xent_pieces={pieces}")
    t = Xent(200, 96, 1900, dtype, seed=2, pieces=pieces)
    t.backward()
    t.check_backward()


def test_pieces_by_size():
    """dz of 16384 x 9001 bf16 is more than a piece holds."""
    t = Xent(16384, 32, 9001, "bf16", seed=3, pieces=4)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("tile", range(4))
@pytest.mark.parametrize("splits", [1, 3])
def test_every_tile(monkeypatch, tile, splits):
    monkeypatch.setenv("STRIPE_TUNE", f"product_tile={tile},product_splits={splits},xent_pieces=2")
    t = Xent(300, 520, 1100, "bf16", seed=4, pieces=2)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


def test_fp32_in_parts(monkeypatch):
    monkeypatch.setenv("STRIPE_TUNE", "product_tile=1")
    t = Xent(200, 256, 700, "f32", seed=5)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ignored", [0.0, 1.0])
def test_all_rows_and_no_row_count(ignored, dtype):
    t = Xent(100, 64, 300, dtype, ignored=ignored, seed=6)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()
    if ignored:
        assert (t.outs["dx"][1] == 0).all() and (t.outs["dw"][1] == 0).all()


@pytest.mark.parametrize("dloss,dlse", [(False, False), (False, True), (True, False)])
def test_gradients_that_are_not_given(dloss, dlse):
    t = Xent(90, 80, 200, "bf16", dloss=dloss, dlse=dlse, seed=7)
    t.backward()
    t.check_backward()


def test_single_outputs():
    t = Xent(70, 64, 150, "bf16", seed=8)
    t.op.run(t.x, t.w, t.targets, t.loss)
    assert (t.lse == -7.0).all()
    loss = t.loss.clone()
    t.op.run(t.x, t.w, t.targets, lse=t.lse)
    assert torch.equal(loss, t.loss)
    t.check_forward()
    t.op.backward(t.x, t.w, t.targets, t.lse_in(), dloss=t.dloss, dlse=t.dlse, dx=t.outs["dx"][1])
    assert (t.outs["dw"][0] == -7.0).all()
    t.check_backward(("dx",))
    t.op.backward(t.x, t.w, t.targets, t.lse_in(), dloss=t.dloss, dlse=t.dlse, dw=t.outs["dw"][1])
    t.check_backward(("dw",))


def test_no_rows():
    t = Xent(0, 64, 100, "bf16")
    t.forward()
    t.backward()
    assert (t.outs["dw"][1] == 0).all()


def test_many_rows_few_of_which_count():
    """More rows than one pass of the counting has threads for."""
    t = Xent(5000, 16, 40, "f32", ignored=0.97, seed=9)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_logits(dtype):
    """Logits of some hundreds: exponentials of distances only."""
    t = Xent(60, 128, 500, dtype, scale=200.0, seed=10)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


def test_infinities_and_nan_go_the_formulas_way():
    inf = float("inf")
    x = torch.ones(5, 8, device="cuda")
    w = torch.zeros(300, 8, device="cuda")
    w[:, 0] = torch.linspace(-1, 1, 300)
    x[0, 1], w[7, 1] = 1, inf           # z[:, 7] = inf where x[:, 1] > 0
    x[1:, 1] = 0.0                      # 0 inf = NaN
    x[2] = NAN
    targets = torch.tensor([3, 3, 3, 7, -1], dtype=torch.int32, device="cuda")
    loss, lse = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    B.StripeXent(5, 8, 300, "f32").run(x, w, targets, loss, lse)
    assert lse[0] == inf and loss[0] == inf and torch.isnan(lse[1:4]).all() and torch.isnan(loss[1:4]).all() and lse[4] == 0
    w[7, 1], w[:, 2] = 0, -inf          # every logit is minus infinity
    B.StripeXent(5, 8, 300, "f32").run(torch.ones_like(x), w, targets, loss, lse)
    assert (lse[:4] == -inf).all() and torch.isnan(loss[:4]).all()
    w[:, 2] = 0
    w[250:, 2] = -inf                   # classes that are masked out by their weights
    B.StripeXent(5, 8, 300, "f32").run(torch.ones_like(x), w, targets, loss, lse)
    want = torch.logsumexp(w[:250, 0].double(), 0)
    assert (abs(lse[:4].double() - want) <= 64 * U * (1 + want.abs())).all()


def test_gradient_against_differences():
    """d/dt of sum(dloss loss + dlse lse) at (x + t d, W + t e), by differences of the forward pass in fp32: off by h^2 / 6 times the third derivative, at most
    6 |d z|^3-like terms for directions whose dz is of size 1, and by the values' errors over h."""
    rows, cin, classes, h = 50, 32, 200, 2.0 ** -6
    t = Xent(rows, cin, classes, "f32", ignored=0.0, seed=11, scale=1.0)
    t.backward()
    g = torch.Generator(device="cuda").manual_seed(12)
    d, e = torch.randn(rows, cin, generator=g, device="cuda") * 0.3, torch.randn(classes, cin, generator=g, device="cuda") * 0.3 * cin ** -0.5

    def total(s):
        loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        t.op.run((t.x + s * d).contiguous(), (t.w + s * e).contiguous(), t.targets, loss, lse)
        return float((t.dloss.double() * loss.double() + t.dlse.double() * lse.double()).sum())

    slope = float((t.outs["dx"][1].double() * d.double()).sum() + (t.outs["dw"][1].double() * e.double()).sum())
    scale = float((t.dloss.abs() + t.dlse.abs()).sum())
    largest = float(t.z.abs().max())
    assert abs((total(h) - total(-h)) / (2 * h) - slope) <= 6 * scale * h * h / 6 + scale * (cin + 64) * U * (1 + largest) / h


def test_streams_graphs_and_repeats(monkeypatch):
    """The same bits on a stream of its own, from a captured graph (replayed among eager work), and from two handles at once."""
    monkeypatch.setenv("STRIPE_TUNE", "xent_pieces=3")
    t, other = (Xent(300, 128, 1500, "bf16", seed=13, pieces=3) for _ in range(2))
    t.op.set_workspace(torch.empty(t.op.workspace_bytes, dtype=torch.uint8, device="cuda").fill_(0xff))
    lse = t.lse_in()

    def both(s):
        s.forward()
        s.op.backward(s.x, s.w, s.targets, lse, dloss=s.dloss, dlse=s.dlse, dx=s.outs["dx"][1], dw=s.outs["dw"][1])

    def results(s):
        return [s.loss, s.lse, s.outs["dx"][1], s.outs["dw"][1]]

    both(t)
    want = [v.clone() for v in results(t)]
    t.check_forward()
    t.check_backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(other)
    both(t)
    torch.cuda.synchronize()
    for s in (t, other):
        assert all(torch.equal(a, b) for a, b in zip(want, results(s)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(t)
    for _ in range(3):
        for v in results(t):
            v.fill_(-7.0)
        graph.replay()
        both(other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, results(t)))


def test_a_first_call_under_capture_is_refused():
    t = Xent(100, 64, 200, "bf16", seed=14)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(B.StripeError):
            t.forward()
        t.loss.add_(0)
    t.forward()
    t.check_forward()


def test_wrapper_refuses_other_tensors():
    t = Xent(20, 64, 32, "bf16", seed=15)
    for args in ((t.x.float(), t.w, t.targets), (t.x, t.w[:16], t.targets), (t.x, t.w, t.targets.long()), (t.x, t.w, t.targets[:10]), (t.x, t.w, t.targets.cpu())):
        with pytest.raises(ValueError):
            t.op.run(*args, t.loss)
    with pytest.raises(B.StripeError):
        t.op.run(t.x, t.w, t.targets, t.loss, t.loss)
    with pytest.raises(B.StripeError):
        t.op.backward(t.x, t.w, t.targets, t.lse, dx=t.x)


@pytest.mark.parametrize("rows", [300, 20000])
@pytest.mark.parametrize("weights", ["zeros", "tiny", "mixed"])
def test_sizes_of_dloss(weights, rows):
    """dz is divided by the largest dloss before its rounding: whatever that is."""
    t = Xent(rows, 48, 130, "bf16", seed=16)
    t.dloss.mul_({"zeros": 0.0, "tiny": 2.0 ** -120, "mixed": 1.0}[weights])
    if weights == "tiny":
        t.dlse.mul_(2.0 ** -120)
    if weights == "mixed":
        t.dloss.mul_(torch.pow(2.0, torch.arange(rows, device="cuda") % 40 - 20.0))
    t.backward()
    t.check_backward()


def test_a_weight_that_is_not_finite_stays_in_its_row():
    t = Xent(40, 64, 100, "bf16", ignored=0.0, seed=17)
    t.dloss[7], t.dloss[8] = float("inf"), NAN
    t.op.backward(t.x, t.w, t.targets, t.lse_in(), dloss=t.dloss, dlse=t.dlse, dx=t.outs["dx"][1])
    got = t.outs["dx"][1]
    assert not torch.isfinite(got[7:9]).any() and torch.isfinite(got[:7]).all() and torch.isfinite(got[9:]).all()


def test_many_rows():
    """More rows than are counted in one launch, a block without any that counts among them."""
    t = Xent(40000, 16, 70, "bf16", ignored=0.5, seed=18)
    t.targets[2048:5000] = -1
    t.counts[2048:5000] = False
    t.z, t.lse_ref = t.x[t.counts].double() @ t.w.double().t(), None
    t.lse_ref = torch.logsumexp(t.z, 1)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("ignored", [0.0, 0.4, 1.0])
def test_more_tiles_than_compute_units(monkeypatch, ignored):
    """Several tiles of 256 x 256 for each compute unit in all four products; with no row that counts the sums have no terms."""
    monkeypatch.setenv("STRIPE_TUNE", "product_tile=0,product_splits=1")
    t = Xent(4360, 4190 if ignored < 1 else 4200, 4300, "bf16", ignored=ignored, pad=2 if ignored < 1 else 0, seed=19, scale=0.5)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


def test_many_tiles_of_short_sums(monkeypatch):
    """One K tile, a part of one, and two to a tile of outputs."""
    monkeypatch.setenv("STRIPE_TUNE", "product_tile=0,product_splits=1,xent_pieces=2")
    for cin in (8, 64, 136):
        t = Xent(4500, cin, 9500, "bf16", ignored=0.1, seed=20, pieces=2)
        t.forward()
        t.check_forward()
        t.backward()
        t.check_backward()


@pytest.mark.parametrize("rows", [5, 100])
def test_infinities_and_nan_in_slices_of_the_reduction(monkeypatch, rows):
    """Logits that are added up from slices, where rows are read in place and where they are copied."""
    monkeypatch.setenv("STRIPE_TUNE", "product_splits=2")
    inf = float("inf")
    x, w = torch.ones(rows, 512, device="cuda"), torch.zeros(300, 512, device="cuda")
    w[:, 0] = torch.linspace(-1, 1, 300)
    w[7, 300] = inf
    x[1:, 300] = 0.0
    x[2] = NAN
    x[4, 300] = NAN
    targets = torch.full((rows,), 3, dtype=torch.int32, device="cuda")
    targets[4] = -1
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    op = B.StripeXent(rows, 512, 300, "f32")
    op.run(x, w, targets, loss, lse)
    assert lse[0] == inf and loss[0] == inf and torch.isnan(lse[1:4]).all() and torch.isnan(loss[1:4]).all() and lse[4] == 0 and loss[4] == 0
    w[7, 300], w[:, 400] = 0, -inf
    op.run(torch.ones_like(x), w, targets, loss, lse)
    assert (lse[:4] == -inf).all() and torch.isnan(loss[:4]).all()
    w[:, 400] = 0
    w[250:, 400] = -inf
    op.run(torch.ones_like(x), w, targets, loss, lse)
    want = torch.logsumexp(w[:250, 0].double(), 0)
    assert (abs(lse[:4].double() - want) <= 64 * U * (1 + want.abs())).all()


def test_dlse_much_larger_than_dloss():
    """dz is divided by the larger of the two weights: nothing overflows."""
    t = Xent(60, 64, 100, "bf16", seed=21)
    t.dloss.mul_(1e-25)
    t.dlse.mul_(1e20)
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_buffers_beyond_32_bits(dtype):
    """Rows of W and dW 2^20 elements apart, the last of them more than 2^32 elements into its buffer."""
    rows, cin, classes, far = 70, 40, 4200, 1 << 20
    t = Xent(rows, cin, classes, dtype, seed=22)
    w = torch.empty(classes * far, dtype=TYPES[dtype], device="cuda").as_strided((classes, cin), (far, 1))
    dw = torch.empty(classes * far, dtype=TYPES[dtype], device="cuda").as_strided((classes, cin), (far, 1))
    w.copy_(t.w)
    op = B.StripeXent(rows, cin, classes, dtype, w_row=far)
    op.run(t.x, w, t.targets, t.loss, t.lse)
    t.check_forward()
    op.backward(t.x, w, t.targets, t.lse_in(), dloss=t.dloss, dlse=t.dlse, dx=t.outs["dx"][1], dw=dw)
    t.outs["dw"][1].copy_(dw)
    t.check_backward()


@pytest.mark.parametrize("rows", [40, 300])
def test_rows_beyond_32_bits(rows):
    """Rows of x and dx so far apart that the last lies more than 2^32 elements in."""
    cin, classes, far = 40, 90, (1 << 32) // 36
    t = Xent(rows, cin, classes, "bf16", seed=23)
    far = far if rows == 40 else (1 << 32) // 290
    x, dx = (torch.empty(rows * far, dtype=torch.bfloat16, device="cuda").as_strided((rows, cin), (far, 1)) for _ in range(2))
    x.copy_(t.x)
    op = B.StripeXent(rows, cin, classes, "bf16", x_row=far)
    op.run(x, t.w, t.targets, t.loss, t.lse)
    t.check_forward()
    op.backward(x, t.w, t.targets, t.lse_in(), dloss=t.dloss, dlse=t.dlse, dx=dx, dw=t.outs["dw"][1])
    t.outs["dx"][1].copy_(dx)
    t.check_backward()


@pytest.mark.parametrize("rows", [1, 3, 70])
def test_more_classes_than_a_piece_holds(rows):
    """More than 2^19 classes: pieces, however few the rows are."""
    t = Xent(rows, 16, 600011, "bf16", ignored=0.0, seed=24, pieces=2)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


@pytest.mark.parametrize("rows", [40, 333])
@pytest.mark.parametrize("cin,classes", [(777, 1300), (70, 515), (1, 9)])
def test_weights_copied_to_whole_pieces(monkeypatch, rows, cin, classes):
    """bf16 rows that are no multiple of 16 bytes, with strides of their own."""
    monkeypatch.setenv("STRIPE_TUNE", "layers_copy=1")
    t = Xent(rows, cin, classes, "bf16", pad=3, shift=1, seed=25)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()


def test_copied_weights_in_pieces_of_the_vocabulary(monkeypatch):
    monkeypatch.setenv("STRIPE_TUNE", "layers_copy=1,xent_pieces=3")
    t = Xent(300, 333, 2000, "bf16", seed=26, pieces=3)
    t.forward()
    t.check_forward()
    t.backward()
    t.check_backward()
