"""The codes of AdamW's 8-bit states where a value lies next to a code's own: equal to those of the formula with an exact root, whatever the random bits are."""
import numpy as np
import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_adamw import F, mix, step8

pytestmark = pytest.mark.gpu


def beside_codes(top, most, n):
    """n values of at most `top`, a block's largest, whose scaled size is one of fp32's next to c^2, c = 1 .. most - 1: below, at, one, two and three above."""
    inverse = F(F(1) / top) * F(most * most)
    c = np.arange(n) // 8 % (most - 1) + 1
    want = (c * c).astype(F)
    for _ in range(3):
        want = np.where(np.arange(n) % 8 > _, np.nextafter(want, F(np.inf)), want)      # 0: c^2 itself
    want = np.where(np.arange(n) % 8 == 5, np.nextafter((c * c).astype(F), F(0)), want)
    value = (want / inverse).astype(F)
    for step in (F(0), F(np.inf)):       # the product is rounded, too: take a neighbour where it is nearer
        other = np.nextafter(value, step)
        value = np.where(abs(other * inverse - want) < abs(value * inverse - want), other, value)
    return np.minimum(value, top).astype(F)


@pytest.mark.parametrize("top", [1.0, 0.7, 1e-3, 3.3e4])
@pytest.mark.parametrize("most", [127, 255])
def test_values_beside_codes(most, top):
    """b1 = b2 = 0: m is the gradient and the root of v its size.  4 M values, so that every kind of them meets random bits that are all zero or all one."""
    n, seed = 1 << 22, 5
    g = beside_codes(F(top), most, n)
    g[::256] = top
    bits = mix((np.arange(n, dtype=np.uint64) + np.uint64(mix(np.array([seed], dtype=np.uint64))[0])) & np.uint64(0xFFFFFFFF))
    assert ((bits & 0xFFFF) == 0).any() and ((bits >> 16) == 0).any()
    grad = torch.from_numpy(g).cuda()
    p = torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(n // 256, device="cuda"), torch.zeros(n // 256, device="cuda")
    op = B.StripeAdamW([n], states="8bit", betas=(0.0, 0.0))
    op.bind([p], [grad], [m], [v], [ms], [vs])
    op.run(1e-3, 1, seed=seed)
    zeros = [np.zeros(n, dtype=np.int8), np.zeros(n // 256, dtype=F), np.zeros(n, dtype=np.uint8), np.zeros(n // 256, dtype=F)]
    _, _, cm, sm, cv, sv = step8(*zeros, g, 0, seed, betas=(0.0, 0.0))
    for name, got, want in (("m", m, cm), ("v", v, cv), ("m_scale", ms, sm), ("v_scale", vs, sv)):
        off = np.flatnonzero(got.cpu().numpy() != want)
        assert not len(off), (name, len(off), [(int(got[i]), int(want[i]), float(g[i]), hex(bits[i])) for i in off[:5]])


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_the_smallest_eps(states):
    """A gradient of 0 is a step of 0."""
    f32 = states == "f32"
    p, g, ms, vs = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros(2, device="cuda"), torch.zeros(2, device="cuda")
    m, v = (torch.zeros(300, dtype=t, device="cuda") for t in ((torch.float32, torch.float32) if f32 else (torch.int8, torch.uint8)))
    op = B.StripeAdamW([300], states=states, eps=2.0 ** -126)
    op.bind([p], [g], [m], [v], *([] if f32 else [[ms], [vs]]))
    op.run(1e-3, 1)
    assert (p == 1).all()
