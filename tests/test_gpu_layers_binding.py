"""layers.py on the GPU: what autograd would have to record, rows over several axes."""
import pytest

from tests.test_gpu_layers import DEV, Attention, rows_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_tensors_that_require_gradients():
    """Refused where gradients are recorded (an input's would be lost), taken inside no_grad and inside a Function, whose backward is the layer's."""
    from paper_1503_02852_amd import RnnError, layers
    c = Attention(9, 2, 2, 1, 16, 16, "f32")
    c.forward()
    c.backward()
    want, x = c.x["o"].clone(), c.x
    for name in ("q", "k", "v"):
        t = dict(x, **{name: x[name].clone().requires_grad_()})
        with pytest.raises(RnnError, match=name + " requires"):
            c.layer.forward(t["q"], t["k"], t["v"], c.log_decay, x["o"], state=c.state)
        x["o"].zero_()
        with torch.no_grad():
            c.layer.forward(t["q"], t["k"], t["v"], c.log_decay, x["o"], state=c.state)
        assert torch.equal(x["o"], want)
    with pytest.raises(RnnError, match="log_decay requires"):
        c.layer.forward(x["q"], x["k"], x["v"], c.log_decay.clone().requires_grad_(), x["o"], state=c.state)
    rows, gain = torch.randn(4, 32, device=DEV), torch.ones(32, device=DEV, requires_grad=True)
    norm = layers.AddNorm(4, 32, dtype=torch.float32, device=DEV)
    with pytest.raises(RnnError, match="gain requires"):
        norm.forward(rows, torch.empty_like(rows), gain=gain)
    with pytest.raises(RnnError, match="x requires"):
        layers.dropout(rows.clone().requires_grad_(), torch.empty_like(rows), 0.5, 1)

    class Of(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            ctx.save_for_backward(q, k, v)
            return c.layer.forward(q, k, v, c.log_decay, torch.empty_like(x["o"]), state=c.state)

        @staticmethod
        def backward(ctx, do):
            q, k, v = ctx.saved_tensors
            out = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
            c.layer.backward(q, k, v, c.log_decay, do.contiguous(), *out, state=c.state, dstate_out=c.dstate_out)
            return out

    leaves = [x[n].clone().requires_grad_() for n in ("q", "k", "v")]
    y = Of.apply(*leaves)
    assert torch.equal(y, want)
    y.backward(x["do"])
    for leaf, name in zip(leaves, ("dq", "dk", "dv")):
        assert torch.equal(leaf.grad, x[name]), name
