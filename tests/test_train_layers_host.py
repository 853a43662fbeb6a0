"""The C entry points of the gated unit, the cross entropy and AdamW, as far as they go without a GPU: what is refused, before anything is launched."""
import ctypes as C

import pytest

from paper_1903_06498_amd import binding as B

ERR = {name: code for code, name in B.STATUS_NAMES.items()}
A = 1 << 20      # an address that is never followed: every call below is refused before a launch


def _status(call):
    with pytest.raises(B.StripeError) as e:
        call()
    assert e.value.detail
    return e.value.status


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "ERR_INVALID_DESC"), (dict(rows=(1 << 28) + 1), "ERR_INVALID_DESC"), (dict(in_features=0), "ERR_INVALID_DESC"),
    (dict(out_features=0), "ERR_INVALID_DESC"), (dict(out_features=(1 << 23) + 1), "ERR_INVALID_DESC"), (dict(groups=-1), "ERR_INVALID_DESC"),
    (dict(groups=4097), "ERR_INVALID_DESC"), (dict(dtype="i8"), "ERR_UNSUPPORTED"), (dict(x_row=31), "ERR_INVALID_DESC"), (dict(w_row=31), "ERR_INVALID_DESC"),
    (dict(y_row=47), "ERR_INVALID_DESC"), (dict(pre_row=95), "ERR_INVALID_DESC"), (dict(groups=2, w_group=96 * 32 - 1), "ERR_INVALID_DESC"),
    (dict(pre_row=(1 << 40) + 8), "ERR_INVALID_DESC"), (dict(rows=1 << 28, out_features=1 << 20), "ERR_UNSUPPORTED"), (dict(rows=1 << 28), "ERR_UNSUPPORTED"),
    (dict(rows=(1 << 28) - 1), "ERR_UNSUPPORTED"),
])
def test_gated_create_refuses(change, status):
    args = dict(rows=16, in_features=32, out_features=48, dtype="bf16")
    args.update(change)
    assert _status(lambda: B.stripe_gated_create(**args)) == ERR[status]


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), "ERR_INVALID_DESC"), (dict(rows=(1 << 24) + 1), "ERR_INVALID_DESC"), (dict(in_features=0), "ERR_INVALID_DESC"),
    (dict(in_features=(1 << 20) + 1), "ERR_INVALID_DESC"), (dict(classes=0), "ERR_INVALID_DESC"), (dict(classes=(1 << 24) + 1), "ERR_INVALID_DESC"),
    (dict(dtype="i32"), "ERR_UNSUPPORTED"), (dict(x_row=31), "ERR_INVALID_DESC"), (dict(w_row=31), "ERR_INVALID_DESC"),
    (dict(rows=1 << 24, classes=1 << 16), "ERR_UNSUPPORTED"),
])
def test_xent_create_refuses(change, status):
    args = dict(rows=16, in_features=32, classes=48, dtype="bf16")
    args.update(change)
    assert _status(lambda: B.stripe_xent_create(**args)) == ERR[status]


@pytest.mark.parametrize("change,status", [
    (dict(elements=[-1]), "ERR_INVALID_DESC"), (dict(elements=[(1 << 34) + 1]), "ERR_INVALID_DESC"), (dict(weight_decay=[float("nan")]), "ERR_INVALID_DESC"),
    (dict(grads="i8"), "ERR_UNSUPPORTED"), (dict(states="bf16"), "ERR_UNSUPPORTED"), (dict(beta1=1.0), "ERR_INVALID_DESC"), (dict(beta2=-0.1), "ERR_INVALID_DESC"),
    (dict(beta1=float("nan")), "ERR_INVALID_DESC"), (dict(eps=-1.0), "ERR_INVALID_DESC"), (dict(eps=float("inf")), "ERR_INVALID_DESC"),
])
def test_adamw_create_refuses(change, status):
    args = dict(elements=[10], weight_decay=[0.0])
    args.update(change)
    assert _status(lambda: B.stripe_adamw_create(**args)) == ERR[status]
    with pytest.raises(ValueError):
        B.stripe_adamw_create([1, 2], [0.0])


def test_null_arguments_are_refused():
    lib, h = B.lib, C.c_void_p()
    for name in ("gated", "xent"):
        assert getattr(lib, f"stripe_{name}_create")(None, C.byref(h)) == ERR["ERR_NULL"]
        assert getattr(lib, f"stripe_{name}_set_workspace")(None, None, 0) == getattr(lib, f"stripe_{name}_workspace_size")(None, None) == ERR["ERR_NULL"]
        getattr(lib, f"stripe_{name}_destroy")(None)
    assert lib.stripe_gated_run(*[None] * 7) == lib.stripe_gated_backward(*[None] * 9) == lib.stripe_gated_query(None, None) == ERR["ERR_NULL"]
    assert lib.stripe_xent_run(*[None] * 7) == lib.stripe_xent_backward(*[None] * 10) == ERR["ERR_NULL"]
    assert lib.stripe_adamw_create(None, C.byref(h)) == lib.stripe_adamw_bind(None, None) == lib.stripe_adamw_run(None, None, None) == ERR["ERR_NULL"]
    assert lib.stripe_adamw_read(None, None, None, None) == ERR["ERR_NULL"]
    lib.stripe_adamw_destroy(None)
    d = B.stripe_gated_desc_t(1, 8, 8, 0, 2, 5)
    assert lib.stripe_gated_create(C.byref(d), C.byref(h)) == ERR["ERR_INVALID_DESC"] and not h.value


def _calls(h, f, good):
    return lambda **change: f(h, *dict(good, **change).values())


def test_gated_run_and_backward_refuse():
    dense, grouped, f32 = (B.stripe_gated_create(16, 32, 48, t, groups=g) for t, g in (("bf16", 0), ("bf16", 3), ("f32", 0)))
    good = dict(x=A, w=2 * A, offsets=None, y=3 * A, pre=None, stream=None)
    call = _calls(dense, B.lib.stripe_gated_run, good)
    for name in ("x", "w", "y"):
        assert call(**{name: None}) == ERR["ERR_NULL"]
        assert call(**{name: A + 1}) == ERR["ERR_MISALIGNED"] == _calls(f32, B.lib.stripe_gated_run, good)(**{name: A + 2})
    assert call(pre=A + 1) == ERR["ERR_MISALIGNED"]
    assert call(y=A) == call(y=2 * A) == call(pre=A) == call(pre=3 * A) == call(offsets=A) == ERR["ERR_INVALID_DESC"]
    call = _calls(grouped, B.lib.stripe_gated_run, good)
    assert call() == ERR["ERR_NULL"] and call(offsets=A + 2) == ERR["ERR_MISALIGNED"] and call(offsets=3 * A) == ERR["ERR_INVALID_DESC"]
    call = _calls(dense, B.lib.stripe_gated_backward, dict(dy=A, x=2 * A, w=3 * A, pre=4 * A, offsets=None, dx=5 * A, dw=6 * A, stream=None))
    assert call(dx=None, dw=None) == 0                  # nothing asked for
    for name in ("dy", "x", "w", "pre"):
        assert call(**{name: None}) == ERR["ERR_NULL"] and call(**{name: A + 1}) == ERR["ERR_MISALIGNED"]
    assert call(dx=A) == call(dw=4 * A) == call(dx=6 * A) == call(offsets=A) == ERR["ERR_INVALID_DESC"]
    for h in (dense, grouped, f32):
        B.lib.stripe_gated_destroy(h)


def test_xent_run_and_backward_refuse():
    h = B.stripe_xent_create(16, 32, 48, "bf16")
    call = _calls(h, B.lib.stripe_xent_run, dict(x=A, w=2 * A, targets=3 * A, loss=4 * A, lse=5 * A, stream=None))
    assert call(loss=None, lse=None) == 0               # nothing asked for
    for name in ("x", "w", "targets"):
        assert call(**{name: None}) == ERR["ERR_NULL"] and call(**{name: A + 1}) == ERR["ERR_MISALIGNED"]
    assert call(loss=A + 2) == call(lse=A + 2) == ERR["ERR_MISALIGNED"]
    assert call(loss=A) == call(lse=3 * A) == call(loss=5 * A) == ERR["ERR_INVALID_DESC"]
    call = _calls(h, B.lib.stripe_xent_backward, dict(x=A, w=2 * A, targets=3 * A, lse=4 * A, dloss=None, dlse=None, dx=5 * A, dw=6 * A, stream=None))
    assert call(dx=None, dw=None) == 0
    for name in ("x", "w", "targets", "lse"):
        assert call(**{name: None}) == ERR["ERR_NULL"] and call(**{name: A + 1}) == ERR["ERR_MISALIGNED"]
    assert call(dloss=A + 2) == call(dlse=A + 2) == call(dx=A + 1) == ERR["ERR_MISALIGNED"]
    assert call(dx=A) == call(dw=4 * A) == call(dx=6 * A) == call(dlse=5 * A) == ERR["ERR_INVALID_DESC"]
    n = C.c_size_t()
    assert B.lib.stripe_xent_workspace_size(h, C.byref(n)) == 0 and n.value > 0
    assert B.lib.stripe_xent_set_workspace(h, A, n.value - 1) == ERR["ERR_NOMEM"]
    assert B.lib.stripe_xent_set_workspace(h, A + 8, n.value) == ERR["ERR_INVALID_DESC"]
    B.lib.stripe_xent_destroy(h)


def test_adamw_bind_and_run_refuse():
    lib = B.lib

    def tensors(*records):
        return (B.stripe_adamw_tensor_t * len(records))(*records)

    f32, i8 = (B.stripe_adamw_create([10, 0, 20], [0.0] * 3, states=s) for s in ("f32", "8bit"))
    step = B.stripe_adamw_step_t(1e-3, 1, 1.0, 0, None)
    none = (None,) * 7
    one, two = (A, 2 * A, 3 * A, 4 * A, None, None, None), (5 * A, 6 * A, 7 * A, 8 * A, None, None, 9 * A)
    assert lib.stripe_adamw_run(f32, C.byref(step), None) == lib.stripe_adamw_bind(f32, None) == lib.stripe_adamw_run(f32, None, None) == ERR["ERR_NULL"]
    assert lib.stripe_adamw_bind(f32, tensors(one, none, two)) == 0        # a tensor without elements needs no buffers
    for i in range(4):
        for bad, status in ((None, "ERR_NULL"), (A * 20 + 2, "ERR_MISALIGNED"), (A if i else 5 * A, "ERR_INVALID_DESC")):
            assert lib.stripe_adamw_bind(f32, tensors(one[:i] + (bad,) + one[i + 1:], none, two)) == ERR[status], (i, bad)
    assert lib.stripe_adamw_bind(f32, tensors(one, none, two[:6] + (A,))) == ERR["ERR_INVALID_DESC"]
    assert lib.stripe_adamw_bind(f32, tensors(one, none, two[:1] + (2 * A,) + two[2:])) == 0      # two gradients may be one
    assert lib.stripe_adamw_bind(f32, tensors(one[:4] + (10 * A, 11 * A, None), none, two)) == ERR["ERR_INVALID_DESC"]
    assert lib.stripe_adamw_bind(i8, tensors(one, none, two)) == ERR["ERR_NULL"]
    for change in (dict(step=0), dict(step=(1 << 53) + 1), dict(lr=float("nan")), dict(factor=float("inf"))):
        bad = B.stripe_adamw_step_t(*dict(dict(lr=1e-3, step=1, factor=1.0, seed=0, control=None), **change).values())
        assert lib.stripe_adamw_run(f32, C.byref(bad), None) == ERR["ERR_INVALID_DESC"]
    bad = B.stripe_adamw_step_t(1e-3, 1, 1.0, 0, A + 2)
    assert lib.stripe_adamw_run(f32, C.byref(bad), None) == ERR["ERR_MISALIGNED"]
    assert lib.stripe_adamw_read(f32, None, None, None) == ERR["ERR_UNSUPPORTED"] and lib.stripe_adamw_read(i8, None, None, None) == ERR["ERR_NULL"]
    for h in (f32, i8):
        lib.stripe_adamw_destroy(h)
    empty = B.stripe_adamw_create([], [])
    assert lib.stripe_adamw_run(empty, C.byref(step), None) == 0
    lib.stripe_adamw_destroy(empty)


def test_gated_plans_and_workspaces_at_the_edges():
    for args in ((0, 1, 1), (1, 1, 1), (1 << 20, 64, 64), (5, 1 << 24, 3), (5, 3, 1 << 23), (100, 33, 1 << 19)):
        for dtype in ("bf16", "f32"):
            h = B.stripe_gated_create(*args, dtype)
            assert B.stripe_gated_query(h)["workspace_bytes"] >= args[0] * 2 * args[2] * 2
            B.lib.stripe_gated_destroy(h)
    for args in ((0, 1, 1), (1, 1, 1), (1 << 24, 8, 100), (1, 1 << 20, 3), (1, 8, 1 << 24), (70000, 64, 1 << 12)):
        for dtype in ("bf16", "f32"):
            B.lib.stripe_xent_destroy(B.stripe_xent_create(*args, dtype))


def test_xent_query():
    info = B.stripe_linear_info_t()
    h = B.stripe_xent_create(16, 32, 48, "bf16")
    assert B.lib.stripe_xent_query(None, C.byref(info)) == B.lib.stripe_xent_query(h, None) == ERR["ERR_NULL"]
    n = C.c_size_t()
    assert B.lib.stripe_xent_workspace_size(h, C.byref(n)) == 0 and B.stripe_xent_query(h)["workspace_bytes"] == n.value
    B.lib.stripe_xent_destroy(h)
    h = B.stripe_xent_create(0, 32, 48, "f32")
    assert B.stripe_xent_query(h)["workspace_bytes"] == 0
    B.lib.stripe_xent_destroy(h)


@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("tile", range(4))
def test_xent_runs_on_the_tile_that_is_asked_for(monkeypatch, tile, splits):
    """The shapes that the GPU tests force tiles for; the logits' reduction of 9 K tiles in 3 slices, dW's of 5 in one."""
    monkeypatch.setenv("STRIPE_TUNE", f"product_tile={tile},product_splits={splits},xent_pieces=2")
    h = B.stripe_xent_create(300, 520, 1100, "bf16")
    info = B.stripe_xent_query(h)
    shape = ("256x256_s2", "128x256_s3", "64x128_s3", "64x64_s4")[tile]
    slices = "" if splits == 1 else "_k3"
    assert info["forward"] == f"product_stream_nt_bf16_{shape}{slices}" and info["input_grad"] == f"product_stream_nn_bf16_{shape}{slices}"
    assert info["weight_grad"] == f"product_stream_tn_bf16_{shape}"
    B.lib.stripe_xent_destroy(h)


def test_xent_names_parts_and_copies(monkeypatch):
    monkeypatch.setenv("STRIPE_TUNE", "product_tile=1")
    h = B.stripe_xent_create(200, 256, 700, "f32")
    assert all("_parts" in B.stripe_xent_query(h)[name] for name in ("forward", "input_grad", "weight_grad"))
    B.lib.stripe_xent_destroy(h)
    monkeypatch.setenv("STRIPE_TUNE", "layers_copy=1")
    h = B.stripe_xent_create(333, 777, 1300, "bf16")
    info = B.stripe_xent_query(h)
    assert info["forward"].endswith("_copied") and info["input_grad"].endswith("_copied")
    B.lib.stripe_xent_destroy(h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_xent_plans_its_input_gradient_for_all_rows(dtype):
    """As a linear layer does whose gradients come in whole pieces, as dz does: of any number of rows, whether W is read where it lies or copied."""
    for rows in (65, 130, 256, 300, 500, 511, 512, 513, 700, 1000):
        for cin, classes in ((4096, 50001), (1024, 10007), (333, 10007), (2048, 32768), (1023, 30841)):
            if rows * classes * (2 if dtype == "bf16" else 4) > 128 << 20:
                continue          # more than one piece
            whole = (classes + 7) // 8 * 8
            h, lin = B.stripe_xent_create(rows, cin, classes, dtype), B.stripe_linear_create(rows, cin, whole, dtype)
            got, want = B.stripe_xent_query(h)["input_grad"], B.stripe_linear_query(lin)["input_grad"]
            B.lib.stripe_xent_destroy(h)
            B.lib.stripe_linear_destroy(lin)
            if got.endswith("_copied"):
                lin = B.stripe_linear_create(rows, (cin + 7) // 8 * 8, whole, dtype)
                want = B.stripe_linear_query(lin)["input_grad"] + "_copied"
                B.lib.stripe_linear_destroy(lin)
            assert got == want, (rows, cin, classes)


@pytest.mark.parametrize("eps", [2.0 ** -127, 1e-40, 1e-300])
def test_adamw_refuses_an_eps_whose_reciprocal_is_infinite(eps):
    """A gradient of 0 would be a step of 0 times infinity."""
    assert _status(lambda: B.stripe_adamw_create([10], [0.0], eps=eps)) == ERR["ERR_INVALID_DESC"]
    for fine in (0.0, 2.0 ** -126, 1e-8):
        B.lib.stripe_adamw_destroy(B.stripe_adamw_create([10], [0.0], eps=fine))
