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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("T,at", [(2, 1), (4, 3), (5, 4), (33, 31), (64, 63), (70, 40), (150, 100), (150, 149), (2500, 1777)])
def test_frames_on_the_other_side_keep_their_results(T, at, bad, dtype):
    """An infinity or NaN in a frame: outputs and dq of earlier frames, dk and dv of later ones are the same bits as without it, as are the other columns of what
    its value alone goes into; what the definition makes infinite or NaN is not finite."""
    names = ("o", "dq", "dk", "dv")
    for which in ("q", "k", "v", "do"):
        c = Attention(T, 1, 2, 2, 40, 40, dtype, seed=T, carry=False, decays=[-0.01, 0.0])

        def run():
            c.forward()
            c.backward()
            return {n: host(c.x[n]).copy() for n in names}

        clean = run()
        c.x[which][at, 0, 1, 7] = bad
        got = run()
        for name in names:
            a, b = clean[name], got[name]
            assert np.array_equal(a[:, :, 0], b[:, :, 0]), (which, name)
            keep = slice(0, at) if name in ("o", "dq") else slice(at + 1, T)
            assert np.array_equal(a[keep], b[keep]), (which, name)
        if which == "v":
            assert np.array_equal(np.delete(clean["o"], 7, 3), np.delete(got["o"], 7, 3))
        hit = {"q": ("o", slice(at, at + 1), slice(None)), "k": ("o", slice(at, T), slice(None)), "v": ("o", slice(at, T), slice(7, 8)),
               "do": ("dv", slice(0, at + 1), slice(7, 8))}[which]
        assert not np.isfinite(got[hit[0]][hit[1], 0, 1, hit[2]]).any(), which
