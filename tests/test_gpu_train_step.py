"""The layers together, as a training step uses them: norm, gated unit, linear layer onto the residual stream, norm, cross entropy over a vocabulary, all
gradients, AdamW -- against automatic differentiation of the formulas in 64 bits, and captured into a graph against itself.

Tolerance of a gradient, in the 2-norm: each of the chain's ten products and norms adds at most (longest sum + 16) u of what goes through it, in fp32, amplified
at most 8 times by the norms (their slope is 1 / spread, and spreads are above 1/2 here, three of them in a row): 10 (256 + 16) u 8 = 1.3e-3 relative."""
import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import TYPES, U

pytestmark = pytest.mark.gpu
ROWS, WIDTH, HIDDEN, CLASSES = 96, 64, 160, 250
NAMES = ("gamma1", "beta1", "w_in", "w_out", "b_out", "gamma2", "beta2", "head")


class Model:
    def __init__(self, dtype, states="f32", seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        dt = TYPES[dtype]
        f32 = dict(dtype=torch.float32, device="cuda")

        def normal(*shape, scale=1.0):
            return torch.randn(*shape, generator=g, device="cuda") * scale

        shapes = {"gamma1": (WIDTH,), "beta1": (WIDTH,), "w_in": (2 * HIDDEN, WIDTH), "w_out": (WIDTH, HIDDEN), "b_out": (WIDTH,), "gamma2": (WIDTH,),
                  "beta2": (WIDTH,), "head": (CLASSES, WIDTH)}
        self.master = {k: normal(*s, scale=WIDTH ** -0.5) + (1.0 if k.startswith("gamma") else 0.0) for k, s in shapes.items()}
        self.matrices = ("w_in", "w_out", "head")
        # the weights that the layers read: bf16 copies of the matrices that the optimizer keeps, or the fp32 values themselves
        self.used = {k: v.to(dt) if k in self.matrices and dtype == "bf16" else v for k, v in self.master.items()}
        self.grad = {k: torch.zeros(s, dtype=dt if k in self.matrices else torch.float32, device="cuda") for k, s in shapes.items()}
        self.x = normal(ROWS, WIDTH).to(dt)
        self.targets = torch.randint(0, CLASSES, (ROWS,), generator=g, device="cuda").to(torch.int32)
        self.targets[::7] = -100
        self.dloss = torch.full((ROWS,), 1.0 / int((self.targets >= 0).sum()), device="cuda")

        def rows(n, dtype=dt):
            return torch.zeros(ROWS, n, dtype=dtype, device="cuda")

        self.n1, self.h, self.pre, self.y, self.n2 = rows(WIDTH), rows(HIDDEN), rows(2 * HIDDEN), rows(WIDTH), rows(WIDTH)
        self.d_n2, self.d_y, self.d_h, self.d_n1, self.d_x = rows(WIDTH), rows(WIDTH), rows(HIDDEN), rows(WIDTH), rows(WIDTH)
        self.stats = [torch.zeros(ROWS, **f32) for _ in range(4)]
        self.loss, self.lse = torch.zeros(ROWS, **f32), torch.zeros(ROWS, **f32)
        self.norm1, self.norm2 = B.StripeNorm(ROWS, WIDTH, dtype), B.StripeNorm(ROWS, WIDTH, dtype)
        self.gated, self.linear, self.head = B.StripeGated(ROWS, WIDTH, HIDDEN, dtype), B.StripeLinear(ROWS, HIDDEN, WIDTH, dtype), B.StripeXent(ROWS, WIDTH, CLASSES, dtype)
        # one optimizer for each type of gradients
        self.optimizers = []
        for names, grads in ((self.matrices, dtype), (tuple(k for k in NAMES if k not in self.matrices), "f32")):
            sizes = [self.master[k].numel() for k in names]
            opt = B.StripeAdamW(sizes, grads=grads, states=states, weight_decay=[0.1 if k in self.matrices else 0.0 for k in names])
            blocks = [-(-n // 256) for n in sizes]
            m, v = ([torch.zeros(n, dtype=t, device="cuda") for n in sizes] for t in ((torch.int8, torch.uint8) if states == "8bit" else (torch.float32,) * 2))
            scales = [[torch.zeros(b, **f32) for b in blocks] for _ in range(2)] if states == "8bit" else (None, None)
            opt.bind([self.master[k] for k in names], [self.grad[k] for k in names], m, v, *scales,
                     copies=[self.used[k] if self.used[k] is not self.master[k] else None for k in names])
            self.optimizers.append(opt)

    def gradients(self):
        u, g, s = self.used, self.grad, self.stats
        self.norm1.run(self.x, self.n1, u["gamma1"], u["beta1"], s[0], s[1])
        self.gated.run(self.n1, u["w_in"], self.h, pre=self.pre)
        self.linear.run(self.h, u["w_out"], self.y, bias=u["b_out"], residual=self.x)
        self.norm2.run(self.y, self.n2, u["gamma2"], u["beta2"], s[2], s[3])
        self.head.run(self.n2, u["head"], self.targets, self.loss, self.lse)
        self.head.backward(self.n2, u["head"], self.targets, self.lse, dloss=self.dloss, dx=self.d_n2, dw=g["head"])
        self.norm2.backward(self.d_n2, self.y, s[2], s[3], u["gamma2"], dx=self.d_y, dgamma=g["gamma2"], dbeta=g["beta2"])
        self.linear.backward(self.d_y, self.h, u["w_out"], dx=self.d_h, dw=g["w_out"], dbias=g["b_out"])
        self.gated.backward(self.d_h, self.n1, u["w_in"], self.pre, dx=self.d_n1, dw=g["w_in"])
        self.norm1.backward(self.d_n1, self.x, s[0], s[1], u["gamma1"], dx=self.d_x, dgamma=g["gamma1"], dbeta=g["beta1"])

    def step(self, *args, **kw):
        for opt in self.optimizers:
            opt.run(*args, **kw)


def reference(model):
    p = {k: v.double().requires_grad_(True) for k, v in model.used.items()}
    x = model.x.double()

    def norm(x, gamma, beta):
        d = x - x.mean(1, keepdim=True)
        return d / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5) * gamma + beta

    z = norm(x, p["gamma1"], p["beta1"]) @ p["w_in"].t()
    g, u = z[:, :HIDDEN], z[:, HIDDEN:]
    y = (g * torch.sigmoid(g) * u) @ p["w_out"].t() + p["b_out"] + x
    z = norm(y, p["gamma2"], p["beta2"]) @ p["head"].t()
    counts = model.targets >= 0
    t = model.targets.long().clamp(min=0)[:, None]
    loss = (torch.logsumexp(z, 1) - z.gather(1, t)[:, 0])[counts]
    (loss * model.dloss[counts].double()).sum().backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}


def test_gradients_and_two_steps_against_64_bits():
    model = Model("f32")
    state = {k: [torch.zeros_like(v, dtype=torch.float64) for _ in range(2)] for k, v in model.master.items()}
    for t in (1, 2):
        loss, want = reference(model)
        before = {k: v.double() for k, v in model.master.items()}
        model.gradients()
        counts = model.targets >= 0
        assert (model.loss[counts].double() - loss).abs().max() <= 8 * (256 + 16) * U * (1 + loss.abs().max())
        for k in NAMES:
            off = float((model.grad[k].double() - want[k]).norm() / want[k].norm())
            assert off <= 1.3e-3, (k, off)
        model.step(1e-2, t)
        for k in NAMES:      # of the gradients that the step was given
            g, (m, v) = model.grad[k].double(), state[k]
            m.mul_(0.9).add_(0.1 * g)
            v.mul_(0.999).add_(0.001 * g * g)
            q = 1e-2 * m / (1 - 0.9 ** t) / (torch.sqrt(v / (1 - 0.999 ** t)) + 1e-8)
            p = before[k] * (1 - 1e-2 * (0.1 if k in model.matrices else 0.0)) - q
            # m may have cancelled between the steps: at most 10 times its terms' roundings are left, |q| is at most about lr
            assert ((model.master[k].double() - p).abs() <= 4 * U * p.abs() + 64 * U * (q.abs() + 1e-2)).all(), k


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_a_captured_step_is_the_eager_one(states):
    """bf16 with copies, numbers from the device: replay by replay the same bits, with eager work of another model between them."""
    a, b = Model("bf16", states), Model("bf16", states)
    controls = [opt.control(1e-2, 1).cuda() for opt in a.optimizers]
    a.gradients()            # allocates the workspaces
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.gradients()
        for opt, control in zip(a.optimizers, controls):
            opt.run(control=control)
    c = Model("bf16", states)
    eager = [opt.control(1e-2, 1).cuda() for opt in c.optimizers]
    for t in (1, 2, 3):
        for opt, control, other in zip(a.optimizers, controls, eager):
            control.copy_(opt.control(2.0 ** -6, t, seed=t))
            other.copy_(control)
        graph.replay()
        c.gradients()
        for opt, control in zip(c.optimizers, eager):
            opt.run(control=control)
        b.gradients()
        torch.cuda.synchronize()
        for k in NAMES:
            assert torch.equal(a.master[k], c.master[k]) and torch.equal(a.used[k], c.used[k]) and torch.equal(a.grad[k], c.grad[k]), (t, k)
            assert torch.isfinite(a.master[k]).all()
        assert torch.equal(a.loss, c.loss)
        if states == "f32":
            for k in a.matrices:
                assert torch.equal(a.used[k], a.master[k].to(torch.bfloat16))
