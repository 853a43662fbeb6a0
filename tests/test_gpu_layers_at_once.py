"""Calls of one layer that overlap, as far as the header allows it."""
import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import Linear, Norm

pytestmark = pytest.mark.gpu


def test_forward_calls_of_one_handle_on_two_streams(monkeypatch):
    """Calls that need no workspace: the linear layer in one piece, the layer norm."""
    monkeypatch.setenv("STRIPE_TUNE", "product_splits=1")
    c, n = Linear(900, 520, 648, "bf16", act="silu", seed=1), Norm(900, 648, "bf16", seed=2)
    assert "_k" not in c.op.info["forward"]
    streams = [torch.cuda.Stream() for _ in range(2)]
    x = [c.x, c.x * 0.5]
    y, pre = [torch.empty_like(c.outs["y"][1]) for _ in range(2)], [torch.empty_like(c.outs["y"][1]) for _ in range(2)]
    h, mean, rstd = [torch.empty_like(n.y) for _ in range(2)], [torch.empty_like(n.mean) for _ in range(2)], [torch.empty_like(n.rstd) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            c.op.run(x[i], c.w, y[i], bias=c.bias, residual=c.residual, pre=pre[i], stream=s.cuda_stream)
            n.op.run(y[i], h[i], gamma=n.gamma, beta=n.beta, mean=mean[i], rstd=rstd[i], stream=s.cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        got = [t.clone() for t in (y[i], pre[i], h[i], mean[i], rstd[i])]
        c.op.run(x[i], c.w, y[i], bias=c.bias, residual=c.residual, pre=pre[i])
        n.op.run(y[i], h[i], gamma=n.gamma, beta=n.beta, mean=mean[i], rstd=rstd[i])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y[i], pre[i], h[i], mean[i], rstd[i])))
    c.outs["y"][1].copy_(y[0])
    c.outs["pre"][1].copy_(pre[0])
    c.check(["y", "pre"])


@pytest.mark.parametrize("what", ["linear", "experts", "norm"])
def test_two_graphs_of_one_handle_with_workspaces_of_their_own(what):
    """Each recorded after a set_workspace of its own, replayed at the same time, with an eager call that has a third between the rounds."""
    if what == "norm":
        c = Norm(700, 1000, "bf16")
        names = ("dx", "dgamma", "dbeta")

        def call(dy, outs, **kw):
            c.op.backward(dy, c.x, c.mean, c.rstd, gamma=c.gamma, **dict(zip(names, outs)), **kw)

        c.forward()
        like = (c.dx, c.dgamma, c.dbeta)
    else:
        c = Linear(700, 264, 520, "bf16", act="silu", offsets=[0, 300, 300, 700] if what == "experts" else None)
        names = ("dx", "dw", "dbias")

        def call(dy, outs, **kw):
            c.op.backward(dy, c.x, c.w, pre=c.pre_in, offsets=c.offsets, **dict(zip(names, outs)), **kw)

        like = (c.outs["dx"][1], c.outs["dw"][1], c.dbias)
    assert c.op.workspace_bytes > 0
    room = [torch.empty(c.op.workspace_bytes, dtype=torch.uint8, device="cuda") for _ in range(3)]
    dys, outs = [c.dy, c.dy * 0.25], [[torch.empty_like(t) for t in like] for _ in range(3)]
    c.op.set_workspace(room[2])
    want = []
    for dy in dys:
        call(dy, outs[2])
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs[2]])
    graphs = []
    for i in range(2):
        c.op.set_workspace(room[i])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.Stream()):
            call(dys[i], outs[i])
        graphs.append(g)
    c.op.set_workspace(room[2])
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(4):
        for o in outs[0] + outs[1] + outs[2]:
            o.fill_(-7.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        call(dys[1], outs[2], stream=streams[2].cuda_stream)
        torch.cuda.synchronize()
        for got, v in zip(outs, (want[0], want[1], want[1])):
            assert all(torch.equal(a, b) for a, b in zip(got, v))


def test_one_handle_on_rows_that_change_place():
    """Calls on windows of one buffer, one after the other on one stream: nothing is kept by an address."""
    op = B.StripeLinear(40, 64, 72, "f32", x_row=64, y_row=72)
    g = torch.Generator(device="cuda").manual_seed(0)
    w = torch.randn(72, 64, generator=g, device="cuda")
    x, y = torch.randn(200, 64, generator=g, device="cuda"), torch.empty(200, 72, device="cuda")
    for step in range(3):
        x.mul_(-0.5)
        for a in range(0, 200, 40):
            op.run(x[a:a + 40], w, y[a:a + 40])
        torch.cuda.synchronize()
        v = x.double() @ w.double().t()
        tol = 66 * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t())
        assert ((y.double() - v).abs() <= tol + 2.0 ** -24 * (v.abs() + tol)).all(), step
