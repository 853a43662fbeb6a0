"""The input gradient of the cross entropy of a linear head where its reduction over the vocabulary is split: the fewer of the rows count, the more slices it has.
Tolerances: those of test_gpu_xent.py, which do not hang on the order of a sum."""
import pytest
import torch

from tests.test_gpu_xent import Xent

pytestmark = pytest.mark.gpu


def keep(t, count):
    """Leaves `count` of the rows, spread over all of them."""
    rows = t.shape[0]
    kept = torch.zeros(rows, dtype=torch.bool, device="cuda")
    if count:
        kept[torch.linspace(0, rows - 1, count, device="cuda").round().long()] = True
    assert int(kept.sum()) == count
    t.targets[~kept], t.counts, t.z, t.lse_ref = -5, kept, t.z[kept], t.lse_ref[kept]


@pytest.mark.parametrize("count", [0, 1, 2, 63, 64, 65, 127, 129, 150, 200, 256, 257, 299, 300])
@pytest.mark.parametrize("dtype,plan", [("bf16", f"product_tile={tile},product_splits={splits}") for tile in range(4) for splits in (2, 5)] +
                         [("f32", f"product_tile={tile},product_splits={splits}") for tile in (1, 2, 3) for splits in (2, 5)])
def test_any_number_of_rows(monkeypatch, dtype, plan, count):
    """Nothing is written behind the workspace, either, whose size is that of the slices that all rows have."""
    monkeypatch.setenv("STRIPE_TUNE", plan)
    t = Xent(300, 72, 2049, dtype, ignored=0.0, pad=8, seed=count)
    assert "_k" + plan[-1] in t.op.info["input_grad"]
    keep(t, count)
    size = t.op.workspace_bytes
    workspace = torch.full((size + (1 << 20),), 0xff, dtype=torch.uint8, device="cuda")
    t.op.set_workspace(workspace[:size])
    t.backward()
    t.check_backward()
    assert (workspace[size:] == 0xff).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cin", [136, 77])
def test_pieces_of_the_vocabulary(monkeypatch, cin, dtype):
    """The last piece has fewer K tiles than the others, and than slices."""
    monkeypatch.setenv("STRIPE_TUNE", "product_splits=4,xent_pieces=3")
    for count in (300, 170, 40, 1):
        t = Xent(300, cin, 1400, dtype, ignored=0.0, seed=count, pieces=3)
        keep(t, count)
        t.backward()
        t.check_backward()


@pytest.mark.parametrize("copies", [0, 1])
def test_copied_weights(monkeypatch, copies):
    monkeypatch.setenv("STRIPE_TUNE", f"product_splits=3,layers_copy={copies}")
    for count in (200, 90, 3):
        t = Xent(200, 333, 1500, "bf16", ignored=0.0, seed=count)
        assert t.op.info["input_grad"].endswith("_copied" if copies else "_k3")
        keep(t, count)
        t.backward()
        t.check_backward()


def test_a_graph_whose_rows_change():
    """A captured pass follows the targets that it finds when it is replayed."""
    t, other = (Xent(512, 520, 9001, "bf16", ignored=0.0, seed=3) for _ in range(2))
    assert "_k" in t.op.info["input_grad"]
    t.backward()
    graph = torch.cuda.CUDAGraph()
    lse = t.lse_in()
    with torch.cuda.graph(graph):
        t.op.backward(t.x, t.w, t.targets, lse, dloss=t.dloss, dlse=t.dlse, dx=t.outs["dx"][1], dw=t.outs["dw"][1])
    full = (t.targets.clone(), t.z, t.lse_ref)
    for count in (512, 70, 0, 300, 512):
        t.targets.copy_(full[0])
        t.z, t.lse_ref = full[1:]
        keep(t, count)
        graph.replay()
        other.backward()
        torch.cuda.synchronize()
        t.check_backward()


def test_both_passes_on_the_same_handle():
    """The forward pass's slices and the input gradient's lie in the same workspace."""
    t = Xent(130, 1032, 700, "bf16", ignored=0.4, seed=4)
    first = None
    for _ in range(3):
        t.forward()
        t.backward()
        t.check_forward()
        t.check_backward()
        first = first if first is not None else t.outs["dx"][1].clone()
        assert torch.equal(first, t.outs["dx"][1])
