"""Every kernel of the linear layer's products on the GPU, whichever the time model would choose: each tile, in one piece and in three slices of the
reduction, dense and with rows sorted by expert, with reductions that go round the ring of LDS stages several times and end inside a K tile.

Values and tolerances are those of test_gpu_layers.py: sums of n terms within (n + 2) u of the sum of their sizes.  A K tile that is left out,
taken twice or read from the wrong stage is 64 (32) terms of a sum of up to 1816, whose tolerance is about a third of one typical term.
"""
import pytest
import torch

from paper_1903_06498_amd import binding as B
from tests.test_gpu_layers import NAN, U, Linear, untouched, window

pytestmark = pytest.mark.gpu

NAMES = ["y", "pre", "dx", "dw", "dbias"]
KINDS = ("forward", "input_grad", "weight_grad")
# dense: 28 K tiles of 64 in x and dz, 27.4 in dW; three slices of them and, in groups, of 21 still go round each ring
DENSE = dict(rows=1755, cin=1784, cout=1816)
SORTED = dict(rows=3600, cin=1352, cout=1368, offsets=[5, 1500, 1500, 3590])      # (an empty group; rows of none at both ends)
TILES = ["256x256_s2", "128x256_s3", "64x128_s3", "64x64_s4"]


def planned(monkeypatch, tune, what, **kw):
    """A layer made under STRIPE_TUNE; `what`: a part of all three kernels' names."""
    monkeypatch.setenv("STRIPE_TUNE", f"product_few=0,{tune}")
    c = Linear(**kw)
    for kind in KINDS:
        assert what in c.op.info[kind], c.op.info
    return c


def both_ways(c):
    c.forward()
    c.check(["y", "pre"])
    c.backward()
    c.check(["dx", "dw", "dbias"])


def slices(splits):
    return f"_k{splits}" if splits > 1 else ""


@pytest.mark.parametrize("shape", [DENSE, SORTED], ids=["dense", "sorted"])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("tile", range(4))
def test_bf16_tiles(tile, splits, shape, monkeypatch):
    c = planned(monkeypatch, f"product_tile={tile},product_splits={splits}", TILES[tile] + slices(splits), dtype="bf16", act="gelu", seed=tile, **shape)
    assert all(c.op.info[k].startswith("product_stream_") and c.op.info[k].endswith(TILES[tile] + slices(splits)) for k in KINDS), c.op.info
    both_ways(c)


@pytest.mark.parametrize("tile", range(4))
def test_bf16_tiles_without_epilogue_and_with_outputs_at_any_element(tile, monkeypatch):
    """No bias and no residual; then x and W in whole pieces, y, pre, residual, dx and dW one element off."""
    c = planned(monkeypatch, f"product_tile={tile},product_splits=1", TILES[tile], dtype="bf16", bias=False, residual=False, rows=700, cin=712, cout=648)
    both_ways(c)
    c = planned(monkeypatch, f"product_tile={tile},product_splits=1", TILES[tile], dtype="bf16", act="silu", pad=8, rows=700, cin=712, cout=648)
    for name, (_, v) in list(c.outs.items()):
        c.outs[name] = window(tuple(v.shape), v.shape[-1] + 8, v.dtype, 1, -7.0)
    residual = window(tuple(c.residual.shape), c.residual.shape[-1] + 8, c.residual.dtype, 1)[1]
    residual.copy_(c.residual)
    c.residual = residual
    both_ways(c)


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("offsets", [None, [0, 400, 400, 1390]], ids=["dense", "sorted"])
def test_bf16_at_any_alignment(offsets, splits, monkeypatch):
    """Odd sizes: through registers, ten K tiles and more."""
    c = planned(monkeypatch, f"product_splits={splits}", "64x128" + slices(splits), dtype="bf16", act="gelu_tanh", rows=1400, cin=777, cout=853, offsets=offsets, seed=5)
    assert not any("stream" in c.op.info[k] for k in KINDS)
    both_ways(c)


F32 = {"pieces": dict(rows=1000, cin=420, cout=388), "words": dict(rows=1000, cin=421, cout=389), "words_windows": dict(rows=1000, cin=420, cout=388, pad=1, shift=1)}


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("offsets", [None, [3, 400, 400, 960]], ids=["dense", "sorted"])
@pytest.mark.parametrize("where", list(F32))
@pytest.mark.parametrize("tile,what", [(1, "64x128_parts"), (2, "64x128_s3"), (3, "64x64_s4")])
def test_f32_tiles(tile, what, where, offsets, splits, monkeypatch):
    """In three bf16 parts, and with fp32 instructions from whole pieces and from words: 11 to 31 K tiles and five values more."""
    name = what + ("" if tile == 1 or where == "pieces" else "_words") + slices(splits)
    c = planned(monkeypatch, f"product_tile={tile},product_splits={splits}", name, dtype="f32", act="silu", offsets=offsets, seed=tile, **F32[where])
    both_ways(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_far_apart_with_many_k_tiles(dtype, monkeypatch):
    """Strides beyond the 32-bit offsets of loads into LDS, reductions of 11 (5) K tiles and five more: the loop over whole tiles at such strides."""
    c = planned(monkeypatch, "product_splits=1", "product_", dtype=dtype, act="relu", rows=357, cin=357, cout=357, pad=(1 << 20) + 3, seed=8)
    assert not any("stream" in c.op.info[k] for k in KINDS) and (dtype == "bf16" or all(c.op.info[k].endswith("_parts") for k in KINDS))
    both_ways(c)


@pytest.mark.parametrize("splits", [1, 3])
def test_f32_in_parts_with_some_tiles_that_are_computed_again(splits, monkeypatch):
    """Infinities and NaN in the first 64 rows only: the other row tiles' sums come from the parts, and are right; those rows show what the formula has."""
    c = planned(monkeypatch, f"product_tile=1,product_splits={splits}", "parts" + slices(splits), dtype="f32", bias=False, residual=False, rows=300, cin=421, cout=389, seed=3)
    clean_x, clean_dy = c.x.clone(), c.dy.clone()
    c.forward()
    c.backward()
    c.check(NAMES)
    for t in (c.x, c.dy):
        t[3, 5], t[7, 0], t[9, 6] = float("inf"), NAN, float("-inf")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    w, rest = c.w.double(), [i for i in range(300) if i not in (3, 7, 9)]
    for got, a, clean, b in ((c.outs["y"][1], c.x, clean_x, w.t()), (c.outs["dx"][1], c.dy, clean_dy, w)):
        a, clean = a.double(), clean.double()
        v = clean @ b
        tol = (a.shape[1] + 2) * U * (clean.abs() @ b.abs())
        tol = tol + U * (v.abs() + tol)
        assert ((got.double() - v).abs() <= tol)[rest].all()
        assert torch.isnan(got[7]).all()
        assert torch.equal(got[3].sign(), b[5].sign().float()) and torch.isinf(got[3]).all()
        assert torch.equal(got[9].sign(), -b[6].sign().float()) and torch.isinf(got[9]).all()
    # dW: columns 0, 5, 6 of x and rows 0, 5, 6 of dz hold them
    v, terms = clean_dy.double().t() @ clean_x.double(), clean_dy.double().abs().t() @ clean_x.double().abs()
    tol = 302 * U * terms
    tol = tol + U * (v.abs() + tol)
    keep_r, keep_c = ([i for i in range(n) if i not in (0, 5, 6)] for n in (389, 421))
    got = c.outs["dw"][1]
    assert ((got.double() - v).abs() <= tol)[keep_r][:, keep_c].all()
    assert not torch.isfinite(got[[0, 5, 6]]).any() and not torch.isfinite(got[:, [0, 5, 6]]).any()
    for name in ("y", "dx", "dw"):
        assert untouched(*c.outs[name], -7.0)


def test_weight_gradient_of_more_than_two_billion_elements():
    """dW beyond 2^31 elements, on 256 x 256 tiles: its first and last rows."""
    rows, cin, cout = 200, 65544, 32776
    g = torch.Generator(device="cuda").manual_seed(0)
    x, dy = (torch.randn(rows, n, generator=g, device="cuda").to(torch.bfloat16) for n in (cin, cout))
    dw = torch.full((cout, cin), -7.0, dtype=torch.bfloat16, device="cuda")
    op = B.StripeLinear(rows, cin, cout, "bf16")
    assert "256x256" in op.info["weight_grad"]
    op.backward(dy, x, None, dw=dw)
    torch.cuda.synchronize()
    for part in (slice(0, 40), slice(cout - 40, cout)):
        v, terms = dy[:, part].double().t() @ x.double(), dy[:, part].double().abs().t() @ x.double().abs()
        tol = (rows + 2) * U * terms
        assert ((dw[part].double() - v).abs() <= tol + 2.0 ** -8 * (v.abs() + tol)).all()
    assert not (dw == -7.0).all(1).any()
