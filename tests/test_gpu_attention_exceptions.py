"""Linear attention: NaN and infinities, in the decays and in frames."""
import numpy as np
import pytest

from tests.test_gpu_layers import DEV, Attention, host

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [1, 3, 40, 150, 2500])
def test_a_decay_that_is_nan(T, dtype):
    """The head's results are NaN wherever the definition's are, and nowhere else; the other heads' are what they are without it."""
    names = ("o", "dq", "dk", "dv")
    c = Attention(T, 2, 3, 3, 32, 24, dtype, [T, (T + 1) // 2], seed=T, decays=[-0.1, -0.2, 0.0])

    def run():
        c.forward()
        c.backward()
        return {n: host(c.x[n]).copy() for n in names} | {"state_out": host(c.state_out), "dstate": host(c.dstate)}

    clean = run()
    c.decays[1] = c.log_decay[1] = float("nan")
    got = run()
    with np.errstate(invalid="ignore"):
        want = c.oracle() | c.oracle(backward=True)
    for name, x in got.items():
        axis = 2 if name in names else 1
        other = lambda a: np.delete(a, 1, axis)  # noqa: E731
        assert np.array_equal(other(x), other(clean[name])), name
        bad = np.isnan(want[name])
        if name in names:
            for n, last in enumerate(c.lengths_host):
                bad[last:, n] = False
        assert bad.any() or name in ("dk", "dv") and T == 1
        assert np.array_equal(np.isnan(x), bad), name
