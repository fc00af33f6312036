"""Calls of the step after a gradient from torch: tensors that do not stand for one another, graphs of autograd that saved
what is written."""
import pytest
import torch

import paper_2503_12382_amd as reno

pytestmark = pytest.mark.gpu


def operands(shape=(6, 10), dtype=torch.float32):
    g = torch.Generator().manual_seed(3)
    w, d = (torch.randn(shape, generator=g).to(dtype).cuda() for _ in range(2))
    return dict(params=[w], grads=[d], exp_avg=[torch.zeros(shape, device="cuda")], exp_avg_sq=[torch.zeros(shape, device="cuda")],
                steps=torch.zeros(2, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("which", ["params", "grads", "exp_avg", "exp_avg_sq", "master"])
def test_tensors_of_another_shape_are_refused(which):
    """As many elements in another shape, a transposed gradient say, are other elements."""
    for shape in ((10, 6), (6, 5, 2), (60, 1), (1, 60)):
        a = operands(dtype=torch.bfloat16)
        a["master"] = [a["params"][0].float()]
        before = a["params"][0].clone()
        a[which] = [a[which][0].reshape(shape).contiguous()]
        with pytest.raises(ValueError, match="shape"):
            reno.adamw_step(**a)
        assert torch.equal(a["params"][0].flatten(), before.flatten()) and a["steps"].tolist() == [0, 0]
    # one flat operand among others does not hide two that differ
    a = operands()
    a["params"], a["exp_avg"] = [a["params"][0].flatten()], [torch.zeros(10, 6, device="cuda")]
    with pytest.raises(ValueError, match="shape"):
        reno.adamw_step(**a)
    a = operands(dtype=torch.bfloat16)
    a["params"], a["master"] = [a["params"][0].flatten()], [torch.zeros(10, 6, device="cuda")]
    with pytest.raises(ValueError, match="shape"):
        reno.adamw_step(**a)


def test_outputs_of_another_shape_are_refused():
    x, n = torch.ones(6, 10, device="cuda"), torch.ones((), device="cuda")
    for shape in ((10, 6), (6, 5, 2), (60, 1)):
        out = torch.zeros(shape, device="cuda")
        with pytest.raises(ValueError, match="shape"):
            reno.clip_grads([x], n, 1.0, out=[out])
        assert bool((out == 0).all())
    with pytest.raises(ValueError):
        reno.clip_grads([x], n, 1.0, out=[torch.zeros(59, device="cuda")])


def test_flat_tensors_stand_for_any_shape():
    """Buffers of all of a tensor's elements in order, as programs with flat state keep them."""
    a, b = operands(), operands()
    for name in ("grads", "exp_avg", "exp_avg_sq"):
        b[name] = [b[name][0].flatten()]
    c = operands()
    c["params"] = [c["params"][0].flatten()]
    for x in (a, b, c):
        reno.adamw_step(**x, lr=0.1)
    for x in (b, c):
        for name in ("params", "exp_avg", "exp_avg_sq"):
            assert torch.equal(x[name][0].flatten(), a[name][0].flatten())
    one = reno.clip_grads(a["grads"], torch.tensor(4.0, device="cuda"), 1.0, out=[torch.zeros(60, device="cuda")])
    assert torch.equal(one[0].view(6, 10), a["grads"][0] / 4)
    # a scalar, and one element
    s = operands(())
    s["grads"], s["exp_avg"] = [s["grads"][0].view(1)], [torch.zeros(1, 1, device="cuda")]
    reno.adamw_step(**s)
    assert s["steps"].tolist() == [1, 0]


def test_what_is_written_counts_as_changed():
    """Autograd's error, and no wrong gradient, where a graph saved weights that a step has moved since."""
    a = operands()
    w = a["params"][0].requires_grad_()
    y = (w * w).sum()
    y.backward(retain_graph=True)
    a["grads"] = [w.grad]
    reno.adamw_step(**a)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    (w * w).sum().backward()          # a new graph
    x = torch.ones(6, 10, device="cuda")
    h = torch.ones(6, 10, device="cuda", requires_grad=True)
    y = (h * x).sum()
    reno.clip_grads([x], torch.ones((), device="cuda"), 0.5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    # what is written, and nothing else
    a = operands(dtype=torch.bfloat16)
    a["master"] = [a["params"][0].float()]
    n = reno.grad_norm(a["grads"])
    flat = [t for k in ("params", "exp_avg", "exp_avg_sq", "master") for t in a[k]] + [a["steps"]]
    before = [t._version for t in flat], a["grads"][0]._version, n._version
    reno.adamw_step(**a, norm=n, max_norm=1.0)
    assert all(t._version > b for t, b in zip(flat, before[0]))
    assert (a["grads"][0]._version, n._version) == before[1:]
    out = [torch.zeros(6, 10, dtype=torch.bfloat16, device="cuda")]
    at = out[0]._version
    reno.clip_grads(a["grads"], n, 1.0, out=out)
    assert out[0]._version > at and a["grads"][0]._version == before[1]


def test_tensors_of_inference_mode():
    """They have no version: a step takes them in that mode and outside it."""
    with torch.inference_mode():
        a = operands()
    b = operands()
    b["steps"] = a["steps"].clone()
    with torch.inference_mode():
        reno.adamw_step(**a, lr=0.1)
    reno.adamw_step(**a, lr=0.1)
    reno.clip_grads(a["grads"], torch.ones((), device="cuda"), 0.5)
    for _ in range(2):
        reno.adamw_step(**b, lr=0.1)
    reno.clip_grads(b["grads"], torch.ones((), device="cuda"), 0.5)
    assert all(torch.equal(a[k][0], b[k][0]) for k in ("params", "exp_avg", "exp_avg_sq", "grads"))
