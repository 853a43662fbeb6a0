"""The layers' C entry points and their Python wrappers, as far as they go without a GPU: what is refused, and that a refusal launches
nothing (there is nothing to launch on here)."""
import ctypes as C

import pytest
import torch

from paper_1903_06498_amd import binding as B

ERR = {name: code for code, name in B.STATUS_NAMES.items()}


def _status(call, *args):
    with pytest.raises(B.StripeError) as e:
        call(*args)
    assert e.value.detail
    return e.value.status


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "ERR_INVALID_DESC"), (dict(rows=(1 << 28) + 1), "ERR_INVALID_DESC"), (dict(in_features=0), "ERR_INVALID_DESC"),
    (dict(out_features=0), "ERR_INVALID_DESC"), (dict(in_features=(1 << 24) + 1), "ERR_INVALID_DESC"), (dict(groups=-1), "ERR_INVALID_DESC"),
    (dict(groups=4097), "ERR_INVALID_DESC"), (dict(dtype="i8"), "ERR_UNSUPPORTED"), (dict(dtype="i32"), "ERR_UNSUPPORTED"),
    (dict(x_row=31), "ERR_INVALID_DESC"), (dict(w_row=31), "ERR_INVALID_DESC"), (dict(y_row=47), "ERR_INVALID_DESC"), (dict(x_row=-40), "ERR_INVALID_DESC"),
    (dict(groups=2, w_group=48 * 32 - 1), "ERR_INVALID_DESC"), (dict(x_row=(1 << 40) + 8), "ERR_INVALID_DESC"),
    (dict(rows=1 << 28, out_features=1 << 20), "ERR_UNSUPPORTED"),
])
def test_linear_create_refuses(change, status):
    args = dict(rows=16, in_features=32, out_features=48, dtype="bf16")
    args.update(change)
    assert _status(lambda: B.stripe_linear_create(**args)) == ERR[status]


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "ERR_INVALID_DESC"), (dict(rows=(1 << 30) + 1), "ERR_INVALID_DESC"), (dict(features=0), "ERR_INVALID_DESC"),
    (dict(dtype="i8"), "ERR_UNSUPPORTED"), (dict(eps=-1e-5), "ERR_INVALID_DESC"), (dict(eps=float("nan")), "ERR_INVALID_DESC"),
    (dict(eps=float("inf")), "ERR_INVALID_DESC"), (dict(eps=1e300), "ERR_INVALID_DESC"), (dict(x_row=31), "ERR_INVALID_DESC"), (dict(y_row=31), "ERR_INVALID_DESC"),
])
def test_norm_create_refuses(change, status):
    args = dict(rows=16, features=32, dtype="f32")
    args.update(change)
    assert _status(lambda: B.stripe_norm_create(**args)) == ERR[status]


def test_unknown_activation_and_null_arguments_are_refused():
    d, h = B.stripe_linear_desc_t(1, 8, 8, 0, 2, 5, 0, 0, 0, 0), C.c_void_p()
    assert B.lib.stripe_linear_create(C.byref(d), C.byref(h)) == ERR["ERR_INVALID_DESC"] and not h.value
    d.activation = -1
    assert B.lib.stripe_linear_create(C.byref(d), C.byref(h)) == ERR["ERR_INVALID_DESC"]
    assert B.lib.stripe_linear_create(None, C.byref(h)) == ERR["ERR_NULL"]
    assert B.lib.stripe_linear_create(C.byref(d), None) == ERR["ERR_NULL"]
    assert B.lib.stripe_norm_create(None, C.byref(h)) == ERR["ERR_NULL"]
    for f, n in ((B.lib.stripe_linear_run, 8), (B.lib.stripe_linear_backward, 9), (B.lib.stripe_norm_run, 7), (B.lib.stripe_norm_backward, 9)):
        assert f(*[None] * (n + 1)) == ERR["ERR_NULL"]
    assert B.lib.stripe_linear_set_workspace(None, None, 0) == B.lib.stripe_norm_set_workspace(None, None, 0) == ERR["ERR_NULL"]
    assert B.lib.stripe_linear_workspace_size(None, None) == B.lib.stripe_norm_workspace_size(None, None) == ERR["ERR_NULL"]
    assert B.lib.stripe_linear_query(None, None) == ERR["ERR_NULL"]
    B.lib.stripe_linear_destroy(None)
    B.lib.stripe_norm_destroy(None)


# addresses that are never followed: every call below is refused before a launch
A = 1 << 20


def _linear(**kw):
    return B.stripe_linear_create(16, 32, 48, kw.pop("dtype", "bf16"), **kw)


def test_linear_run_refuses():
    run = B.lib.stripe_linear_run
    dense, grouped, f32 = _linear(), _linear(groups=3), _linear(dtype="f32")
    good = dict(x=A, w=A, bias=None, residual=None, offsets=None, y=A, pre=None, stream=None)

    def call(h, **change):
        return run(h, *dict(good, **change).values())

    for name in ("x", "w", "y"):
        assert call(dense, **{name: None}) == ERR["ERR_NULL"]
    for name in ("x", "w", "y", "residual", "pre"):
        assert call(dense, **{name: A + 1}) == ERR["ERR_MISALIGNED"]
        assert call(f32, **{name: A + 2}) == ERR["ERR_MISALIGNED"]
    assert call(dense, bias=A + 2) == ERR["ERR_MISALIGNED"]
    assert call(dense, offsets=A) == ERR["ERR_INVALID_DESC"]
    assert call(grouped) == ERR["ERR_NULL"]
    assert call(grouped, offsets=A + 2) == ERR["ERR_MISALIGNED"]
    for h in (dense, grouped, f32):
        B.lib.stripe_linear_destroy(h)


def test_linear_backward_refuses():
    backward = B.lib.stripe_linear_backward
    plain, act, grouped = _linear(), _linear(activation="silu"), _linear(groups=3)
    good = dict(dy=A, x=A, w=A, pre=A, offsets=None, dx=A, dw=A, dbias=A, stream=None)

    def call(h, **change):
        return backward(h, *dict(good, **change).values())

    assert call(plain, dx=None, dw=None, dbias=None) == 0                       # nothing asked for
    for name in ("dy", "x", "w"):
        assert call(plain, **{name: None}) == ERR["ERR_NULL"]
    assert call(act, pre=None) == ERR["ERR_NULL"]
    for name in ("dy", "x", "w", "pre", "dx", "dw"):
        assert call(act, **{name: A + 1}) == ERR["ERR_MISALIGNED"]
    assert call(act, dbias=A + 2) == ERR["ERR_MISALIGNED"]
    assert call(grouped) == ERR["ERR_NULL"] and call(plain, offsets=A) == ERR["ERR_INVALID_DESC"]
    for h in (plain, act, grouped):
        B.lib.stripe_linear_destroy(h)


def test_norm_refuses():
    h = B.stripe_norm_create(16, 32, "bf16")
    run, back = B.lib.stripe_norm_run, B.lib.stripe_norm_backward
    assert run(h, None, None, None, A, None, None, None) == run(h, A, None, None, None, None, None, None) == ERR["ERR_NULL"]
    assert run(h, A + 1, None, None, A, None, None, None) == run(h, A, A + 2, None, A, None, None, None) == ERR["ERR_MISALIGNED"]
    assert run(h, A, None, None, A, A + 1, None, None) == ERR["ERR_MISALIGNED"]
    assert back(h, A, A, None, A, A, None, None, None, None) == 0               # nothing asked for
    for i in (1, 2, 4, 5):
        args = [h, A, A, None, A, A, A, None, None, None]
        args[i] = None
        assert back(*args) == ERR["ERR_NULL"]
    assert back(h, A, A, None, A, A, A + 1, None, None, None) == back(h, A, A, None, A, A, A, A + 2, None, None) == ERR["ERR_MISALIGNED"]
    B.lib.stripe_norm_destroy(h)


def test_no_rows_is_no_work():
    h = B.stripe_linear_create(0, 32, 48, "bf16")
    assert B.lib.stripe_linear_run(h, *[None] * 8) == 0
    B.lib.stripe_linear_destroy(h)
    h = B.stripe_norm_create(0, 32, "bf16")
    assert B.lib.stripe_norm_run(h, *[None] * 7) == 0
    B.lib.stripe_norm_destroy(h)


@pytest.mark.parametrize("make", [lambda: B.StripeLinear(512, 256, 384, "bf16", activation="gelu"), lambda: B.StripeNorm(512, 256, "bf16")])
def test_workspaces_are_checked(make):
    h = make()
    assert h.workspace_bytes > 0 and h.workspace_bytes % 256 == 0
    set_ws = getattr(B.lib, f"stripe_{h._name}_set_workspace")
    assert set_ws(h.handle, A, h.workspace_bytes) == 0
    assert set_ws(h.handle, A, h.workspace_bytes - 1) == ERR["ERR_NOMEM"]
    assert set_ws(h.handle, A + 16, h.workspace_bytes) == ERR["ERR_INVALID_DESC"]
    assert set_ws(h.handle, None, 0) == 0
    with pytest.raises(ValueError):
        h.set_workspace(torch.empty(h.workspace_bytes, dtype=torch.uint8))      # host memory
    h.close()


def test_wrapper_checks_tensors():
    h = B.StripeLinear(4, 8, 16, "bf16", groups=2, x_row=12)
    shape, strides = h._x
    check = lambda t: h._ptr("x", t, torch.bfloat16, shape, strides, -1)        # noqa: E731  (-1: host tensors, for this test)
    good = torch.empty(4, 12, dtype=torch.bfloat16)[:, :8]
    assert check(good) == good.data_ptr() and check(None) is None
    for bad in (good.float(), torch.empty(4, 8, dtype=torch.bfloat16), good[:3], torch.empty(8, 4, dtype=torch.bfloat16).t()):
        with pytest.raises(ValueError, match="x: expected"):
            check(bad)
    with pytest.raises(ValueError):
        h._ptr("x", good, torch.bfloat16, shape, strides, 0)                    # another device
    assert h._w == ((2, 16, 8), (128, 8, 1)) and h._b == ((2, 16), (16, 1)) and h._o == ((3,), (1,))
    one = B.StripeLinear(1, 8, 16, "bf16", x_row=64)                            # the stride of a single row does not matter
    assert one._ptr("x", torch.empty(1, 8, dtype=torch.bfloat16), torch.bfloat16, *one._x, -1)


@pytest.mark.parametrize("change", [dict(rows=1 << 20, x_row=1 << 40), dict(rows=1 << 20, y_row=1 << 40), dict(out_features=1 << 18, w_row=1 << 40),
                                    dict(groups=4096, w_group=1 << 60), dict(groups=4096, w_row=1 << 40, out_features=1 << 10)])
def test_buffers_beyond_64_bit_offsets_are_refused(change):
    args = dict(rows=16, in_features=32, out_features=48, dtype="bf16")
    args.update(change)
    assert _status(lambda: B.stripe_linear_create(**args)) == ERR["ERR_INVALID_DESC"]
    for name in ("x_row", "y_row"):
        assert _status(lambda: B.stripe_norm_create(1 << 20, 32, "f32", **{name: 1 << 40})) == ERR["ERR_INVALID_DESC"]


def test_outputs_that_are_inputs_are_refused():
    """Every buffer at an address of its own but for one pair."""
    spread = lambda names: {n: (i + 1) << 20 for i, n in enumerate(names)}      # noqa: E731
    lin, norm, strided = _linear(activation="silu"), B.stripe_norm_create(16, 32, "bf16"), B.stripe_norm_create(16, 32, "bf16", y_row=40)

    def check(call, handle, names, pairs):
        for a, b in pairs:
            args = spread(names)
            if "offsets" in args:
                args["offsets"] = None
            args[a] = args[b]
            assert call(handle, *args.values(), None) == ERR["ERR_INVALID_DESC"], (a, b)

    check(B.lib.stripe_linear_run, lin, ("x", "w", "bias", "residual", "offsets", "y", "pre"), [("y", "x"), ("y", "w"), ("pre", "x"), ("pre", "y"), ("pre", "residual")])
    check(B.lib.stripe_linear_backward, lin, ("dy", "x", "w", "pre", "offsets", "dx", "dw", "dbias"),
          [("dx", "dy"), ("dx", "x"), ("dx", "pre"), ("dw", "w"), ("dw", "dx"), ("dbias", "dw")])
    check(B.lib.stripe_norm_run, norm, ("x", "gamma", "beta", "y", "mean", "rstd"), [("y", "gamma"), ("mean", "rstd"), ("mean", "x"), ("rstd", "y")])
    check(B.lib.stripe_norm_run, strided, ("x", "gamma", "beta", "y", "mean", "rstd"), [("y", "x")])
    check(B.lib.stripe_norm_backward, norm, ("dy", "x", "gamma", "mean", "rstd", "dx", "dgamma", "dbeta"),
          [("dx", "dy"), ("dx", "x"), ("dgamma", "gamma"), ("dgamma", "dbeta"), ("dbeta", "mean")])
    B.lib.stripe_linear_destroy(lin)
    for h in (norm, strided):
        B.lib.stripe_norm_destroy(h)


def test_a_workspace_of_another_device_is_refused():
    h = B.StripeNorm(512, 256, "bf16")

    class Elsewhere:
        device = "cuda:1"

        def get_device(self):
            return 1

    h._device, h._ws = lambda: 0, Elsewhere()
    with pytest.raises(ValueError, match="workspace is on"):
        h.run(None, None)
    with pytest.raises(ValueError, match="workspace is on"):
        h.backward(None, None, None, None)
    h._ws = None
    h.close()


def test_few_rows_run_on_their_kernel_where_a_launch_holds_them():
    forward = lambda *a, **kw: B.StripeLinear(*a, **kw).info["forward"]                            # noqa: E731
    assert "rows" in forward(1, 1024, 1024, "f32") and "rows" in forward(8, 1024, 1024, "bf16", groups=8)
    assert "rows" not in forward(65, 1024, 1024, "f32") and "rows" not in forward(1000, 1024, 1024, "bf16", groups=8)
    # 4096 groups of 16 rows at most, 2^17 / 16 columns: more than 2^32 lanes
    assert "rows" not in forward(4096, 8, 1 << 17, "bf16", groups=4096)


@pytest.mark.parametrize("splits", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tile", [1, 2, 3])
def test_the_number_of_slices_can_be_chosen(tile, dtype, splits, monkeypatch):
    """STRIPE_TUNE's product_splits decides, whatever the time model says; one piece where a reduction has too few K tiles for it."""
    monkeypatch.setenv("STRIPE_TUNE", f"product_few=0,product_tile={tile},product_splits={splits}")
    name = f"_k{splits}" if splits > 1 else ""
    for kernel in list(B.StripeLinear(1400, 1352, 1368, dtype, groups=2).info.values())[:3] + list(B.StripeLinear(700, 520, 904, dtype).info.values())[:3]:
        assert kernel.endswith(name) and ("_k" in kernel) == (splits > 1), kernel
    assert not any("_k" in k for k in list(B.StripeLinear(60, 56, 48, "bf16").info.values())[:3])


@pytest.mark.parametrize("features", [16384, 16385, 20000, 1 << 17, 1 << 20, (1 << 22) + 3, 1 << 24])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_norms_workspace_stays_small(dtype, features):
    """The column sums that the backward pass leaves between its launches, whatever the shape: at most 256 rows of 16384 features, or 1024 strips."""
    for rows in (1, 255, 256, 1 << 20):
        h = B.StripeNorm(rows, features, dtype)
        assert h.workspace_bytes <= 256 * 2 * 16384 * 4, (rows, h.workspace_bytes)
        h.close()
