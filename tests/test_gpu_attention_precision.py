"""Linear attention: the bits of a result do not hang on what else the call is asked for."""
import pytest

from tests.test_gpu_layers import Attention

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("T", [20, 64, 200])
def test_the_same_bits_whatever_else_is_asked_for(T):
    """Outputs with and without the last state, gradients with and without the state's, all of them in one segment."""
    c = Attention(T, 1, 2, 1, 64, 64, "bf16", seed=3)
    x = c.x
    c.forward()
    c.backward()
    o = torch.full_like(x["o"], c.MARK)
    c.layer.forward(x["q"], x["k"], x["v"], c.log_decay, o, state=c.state)
    assert torch.equal(o, x["o"])
    with_state = {n: torch.full_like(x[n], c.MARK) for n in ("dq", "dk", "dv")}
    c.layer.backward(x["q"], x["k"], x["v"], c.log_decay, x["do"], **with_state, state=c.state, dstate_out=c.dstate_out)
    assert all(torch.equal(with_state[n], x[n]) for n in with_state)
    for n in with_state:
        alone = torch.full_like(x[n], c.MARK)
        c.layer.backward(x["q"], x["k"], x["v"], c.log_decay, x["do"], **{n: alone}, state=c.state, dstate_out=c.dstate_out)
        assert torch.equal(alone, x[n]), n
